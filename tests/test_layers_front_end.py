"""The Python front end of the layers beside the transducer loss, without a GPU: what it calls when, and what it refuses.  The library's calls are replaced by
records of them, the tensors lie in host memory."""
import pytest
import torch

from paper_2211_16270_amd import binding as Bd

REAL = Bd.lib


class _Library:
    """The library with its calls that launch something recorded instead (all succeed)"""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_workspace_bytes"):
            return getattr(REAL(), name)
        return lambda *args: self.calls.append((name, args)) or 0


class _Stream:
    """Stands for the block in which the stream of a call is the current one"""
    active = False

    def __init__(self, device, stream):
        pass

    def __enter__(self):
        _Stream.active = True

    def __exit__(self, *exc):
        _Stream.active = False


@pytest.fixture
def library(monkeypatch):
    fake = _Library()
    monkeypatch.setattr(Bd, "lib", lambda: fake)
    monkeypatch.setattr(Bd, "_CallOn", _Stream)
    monkeypatch.setattr(Bd, "_stream_handle", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(Bd, "_layer_dtype", lambda x, W, K: Bd.RNNT_BF16 if x.dtype == torch.bfloat16 else Bd.RNNT_F32)
    return fake


def _off(*shape, dtype=torch.bfloat16):
    """A tensor that starts off a 16-byte boundary"""
    n = 1
    for s in shape:
        n *= s
    t = torch.zeros(n + 1, dtype=dtype)[1:].view(shape)
    assert t.data_ptr() % 16 != 0
    return t


def test_copies_of_unaligned_tensors_are_made_on_the_calls_stream(library, monkeypatch):
    clone, where = torch.Tensor.clone, []

    def recorded(self, *args, **kw):
        where.append(_Stream.active)
        return clone(self, *args, **kw)

    monkeypatch.setattr(torch.Tensor, "clone", recorded)
    x, W, b, y, s = _off(5, 8), _off(8, 24), _off(24), _off(5, 24), _off(5, 24, dtype=torch.float16)
    lab = torch.zeros(5, dtype=torch.int32)
    for call, copies in ((lambda: Bd.run_linear_fwd(x, W, b, "silu", y), 4), (lambda: Bd.run_linear_bwd(x, W, y, "silu", s), 4),
                         (lambda: Bd.run_ce_fwd(x, W, b, lab), 3), (lambda: Bd.run_ce_fwd_bwd(x, W, b, lab), 3)):
        where.clear()
        call()
        assert where == [True] * copies
    assert [name for name, _ in library.calls] == ["rnnt_linear_fwd", "rnnt_linear_bwd", "rnnt_ce_loss_fwd", "rnnt_ce_loss_fwd_bwd"]


@pytest.mark.parametrize("x_type,b_type,bits", [(torch.float32, torch.bfloat16, 0), (torch.float32, torch.float32, 0), (torch.bfloat16, torch.bfloat16, 3),
                                                (torch.bfloat16, torch.float32, 1)])
def test_summed_loss_scales_gradients_of_the_librarys_types(library, monkeypatch, x_type, b_type, bits):
    """The descriptor of rnnt_ce_loss_scale is one the library takes, whatever the bias' type; the leaves get gradients of their own types."""
    from paper_2211_16270_amd import autograd as A
    seen = []
    monkeypatch.setattr(Bd, "rnnt_ce_loss_scale", lambda desc, *a, **kw: seen.append(
        (desc.dtype, desc.param_grads_bf16, REAL().rnnt_ce_loss_scale(desc, None, None, None, None, None))) or 0)
    x, W, b = torch.zeros(5, 8, dtype=x_type), torch.zeros(8, 24, dtype=x_type), torch.zeros(24, dtype=b_type)
    leaves = [t.requires_grad_() for t in (x, W, b)]
    A.rnnt_ce_loss(*leaves, torch.zeros(5, dtype=torch.int32)).backward()
    # (a factor of NULL is what the library complains of last)
    assert seen == [(Bd.RNNT_BF16 if x_type == torch.bfloat16 else Bd.RNNT_F32, bits, Bd.STATUS_NAMES.index("RNNT_ERR_NULL"))]
    assert all(t.grad.dtype == t.dtype and t.grad.shape == t.shape for t in leaves)


def test_scaling_refuses_gradients_that_do_not_fit_together(library):
    f = torch.ones(())
    t = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)
    half = torch.float16
    for dx, dW, db in ((t(5, 8, dtype=half), t(8, 24), None), (t(5, 8), t(8, 24, dtype=half), None), (t(5, 8), t(8, 24), t(24, dtype=half)),      # types
                       (t(5, 8), t(8, 24), t(23)), (t(5, 7), t(8, 24), None), (t(5, 8), t(8 * 24), None), (t(5, 8), t(8, 24), t(24, 1)),            # shapes
                       (t(8, 5).t(), t(8, 24), None), (t(5, 8), t(8, 48)[:, ::2], None), (t(5, 8), t(24, 8).t(), None), (t(5, 8), t(8, 24), t(48)[::2]),   # strides
                       (t(5, 8), t(8, 24, dtype=torch.bfloat16), None), (t(5, 8), t(8, 24), t(24, dtype=torch.bfloat16)),        # of no descriptor
                       (t(5, 8).to("meta"), t(8, 24), None), (t(5, 8), t(8, 24).to("meta"), None)):                             # devices
        with pytest.raises(ValueError):
            Bd.run_ce_scale(f, dx, dW, db)
    for factor in (torch.ones(2), torch.ones(0), torch.ones((), dtype=torch.float64)):
        with pytest.raises(ValueError):
            Bd.run_ce_scale(factor, t(5, 8), t(8, 24))
    assert library.calls == []
    Bd.run_ce_scale(f, t(5, 8), t(8, 24), t(24))
    Bd.run_ce_scale(torch.ones(1), t(2, 3, 8, dtype=torch.bfloat16), t(8, 24, dtype=torch.bfloat16), t(24))
    Bd.run_ce_scale(f, t(0, 8), t(8, 24))
    assert len(library.calls) == 3


def test_tensors_in_host_memory_are_refused():
    with pytest.raises(ValueError, match="CUDA"):
        Bd.run_ce_total(torch.zeros(4))
    with pytest.raises(ValueError, match="CUDA"):
        Bd.run_ce_scale(torch.ones(()), torch.zeros(5, 8), torch.zeros(8, 24))


def test_a_workspace_of_another_device_is_refused(library):
    x, W, y, lab = torch.zeros(5, 7), torch.zeros(7, 24), torch.zeros(5, 24), torch.zeros(5, dtype=torch.int32)
    ws = Bd.Workspace.__new__(Bd.Workspace)
    ws.buf = torch.empty(1 << 20, dtype=torch.uint8, device="meta")
    for call in (lambda: Bd.run_linear_fwd(x, W, workspace=ws), lambda: Bd.run_linear_bwd(x, W, y, workspace=ws),
                 lambda: Bd.run_ce_fwd(x, W, None, lab, workspace=ws), lambda: Bd.run_ce_fwd_bwd(x, W, None, lab, workspace=ws)):
        with pytest.raises(ValueError, match="workspace"):
            call()
    assert library.calls == []
    ws.buf = torch.empty(1 << 20, dtype=torch.uint8)
    Bd.run_linear_fwd(x, W, workspace=ws)
    assert len(library.calls) == 1


@pytest.mark.parametrize("off", [torch.no_grad, torch.inference_mode])
def test_nothing_is_computed_for_gradients_where_there_are_none(library, off):
    from paper_2211_16270_amd import autograd as A
    x, W, b, Wl, lab = torch.zeros(5, 8), torch.zeros(8, 24), torch.zeros(24), torch.zeros(8, 16), torch.zeros(5, dtype=torch.int32)
    r = torch.zeros(5, 16)
    state = torch.zeros(2, dtype=torch.int64)

    def names(f):
        library.calls.clear()
        out = f()
        return out, [n for n, _ in library.calls]

    def layer():
        return A.rnnt_linear(x, Wl, None, "silu", r, 0.5, state)

    def check(tracked):
        for reduction, evaluated, trained in (("sum", ["rnnt_ce_loss_fwd", "rnnt_ce_loss_total"], ["rnnt_ce_loss_fwd_bwd", "rnnt_ce_loss_total"]),
                                              ("none", ["rnnt_ce_loss_fwd"], ["rnnt_ce_loss_fwd"])):
            loss, called = names(lambda: A.rnnt_ce_loss(x, W, b, lab, reduction=reduction))
            assert called == (trained if tracked else evaluated) and loss.requires_grad == tracked
            assert loss.shape == (() if reduction == "sum" else (5,))
        y, called = names(layer)
        assert called == ["rnnt_linear_fwd"] and y.requires_grad == tracked
        used, saved = (library.calls[0][1][k] for k in (6, 8))                # (rng_used, saved)
        assert (used is not None) == tracked and (saved is not None) == tracked

    check(False)
    for t in (x, W, b, Wl):
        t.requires_grad_()
    check(True)
    with off():
        check(False)
    for t in (x, W, b, Wl):
        t.requires_grad_(False)
    # a residual's gradient is dy: nothing is kept for it
    r.requires_grad_()
    y, _ = names(layer)
    assert y.requires_grad and library.calls[0][1][8] is None
    y.sum().backward()
    assert bool((r.grad == 1).all())


def test_weights_that_want_a_gradient_are_refused(library):
    from paper_2211_16270_amd import autograd as A
    x, W, lab = torch.zeros(5, 8), torch.zeros(8, 24), torch.zeros(5, dtype=torch.int32)
    w = torch.ones(5, requires_grad=True)
    for leaf in (False, True):
        x.requires_grad_(leaf)
        with pytest.raises(ValueError, match="row_weight"):
            A.rnnt_ce_loss(x, W, None, lab, row_weight=w)
    assert library.calls == []
    A.rnnt_ce_loss(x, W, None, lab, row_weight=w.detach())
    with torch.no_grad():
        A.rnnt_ce_loss(x, W, None, lab, row_weight=w)
    # weights by the formula: their gradient is the rows' losses
    (A.rnnt_ce_loss(x, W, None, lab, reduction="none") * w).sum().backward()
    assert w.grad is not None and x.grad is not None
