"""Calls at the edges of the layers beside the transducer loss, on the GPU: empty batches, streams, graphs, evaluation, mixed types."""
import numpy as np
import pytest

from paper_2211_16270_amd import binding as Bd
from tests import layer_oracle as O
from tests.test_gpu_layers import _ce_inputs, _check_ce, _check_linear, _dev, _linear_inputs, _np, _run_ce, _run_linear, _torch

pytestmark = pytest.mark.gpu


# widths whose backward pass needs no workspace where there are no rows (whole tiles, no copies), and one that does
@pytest.mark.parametrize("K,N", [(512, 2048), (8, 64), (24, 40)])
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("activation", ["none", "silu"])
def test_an_empty_batch_has_gradients_of_zero(K, N, bf16, activation):
    torch = _torch()
    dt = torch.bfloat16 if bf16 else torch.float32
    x, dy, W = torch.zeros(0, K, dtype=dt, device="cuda:0"), torch.zeros(0, N, dtype=dt, device="cuda:0"), torch.ones(K, N, dtype=dt, device="cuda:0")
    saved = None if activation == "none" else torch.zeros(0, N, dtype=torch.float16 if bf16 else torch.float32, device="cuda:0")
    for want in (("dx", "dW", "db"), ("db",), ("dW",)):
        for fill in (7.0, -3.0):
            # (what the allocator hands out next is no zeros)
            junk = [torch.full((n,), fill, device="cuda:0") for n in (N, K * N)]
            del junk
            out = Bd.run_linear_bwd(x, W, dy, activation, saved, want=want)
            for k in ("dW", "db"):
                assert (out[k] is None) == (k not in want)
                assert out[k] is None or bool((out[k] == 0).all()), k
    # added to: unchanged
    dW, db = torch.full((K, N), 2.0, device="cuda:0"), torch.full((N,), -1.5, device="cuda:0")
    Bd.run_linear_bwd(x, W, dy, activation, saved, accumulate_into=(dW, db))
    assert bool((dW == 2.0).all()) and bool((db == -1.5).all())
    from paper_2211_16270_amd import autograd as A
    leaves = [x.requires_grad_(), W.requires_grad_(), torch.zeros(N, device="cuda:0", requires_grad=True)]
    junk = torch.full((N,), 5.0, device="cuda:0")
    del junk
    A.rnnt_linear(*leaves, activation=activation).sum().backward()
    assert leaves[0].grad.shape == (0, K) and bool((leaves[1].grad == 0).all()) and bool((leaves[2].grad == 0).all())


def test_unaligned_views_on_a_stream_of_their_own():
    """The caller's stream has waited for the current one, which is then kept busy: copies of views off a 16-byte boundary follow the call's stream alone."""
    torch = _torch()
    i = _linear_inputs(70, 63, 65, True, res=True)
    c = _ce_inputs(70, 63, 65, True, 9)

    def off(a, dtype=torch.bfloat16):
        flat = torch.zeros(a.size + 1, dtype=dtype, device="cuda:0")
        flat[1:] = _dev(a, dtype).reshape(-1)
        return flat[1:].view(a.shape)

    x, W, r, dy, b = (off(i[k]) for k in ("x", "W", "residual", "dy", "b"))
    xc, Wc, lab, w = off(c["x"]), off(c["W"]), _dev(c["labels"], torch.int32), _dev(c["weight"], torch.float32)

    def calls(stream=None):
        f = Bd.run_linear_fwd(x, W, b, "silu", r, save=True, stream=stream)
        g = Bd.run_linear_bwd(x, W, dy, "silu", f["saved"], stream=stream)
        l = Bd.run_ce_fwd(xc, Wc, b, lab, stream=stream)
        o = Bd.run_ce_fwd_bwd(xc, Wc, b, lab, w, stream=stream)
        return [f["y"], f["saved"], *g.values(), l["loss"], *o.values()]

    want = calls()
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda._sleep(20_000_000)
        got = calls(side)
        # (memory that the call's own copies took may be handed out again on this stream)
        junk = [torch.full((n,), float("nan"), dtype=torch.bfloat16, device="cuda:0") for n in (70 * 63, 63 * 65, 70 * 65, 65)]
        side.synchronize()
        torch.cuda.synchronize()
        del junk
        for a, e in zip(got, want):
            assert torch.equal(a, e)


@pytest.mark.parametrize("R,D,V,bits,budget", [(1024, 64, 2048, 3, 4 << 20), (1856, 512, 1024, 3, 18881224), (1291, 685, 1343, 0, 27 << 20),
                                               (1742, 646, 717, 3, 12 << 20), (1130, 559, 898, 0, 15100000)])
def test_cross_entropy_within_budgets(R, D, V, bits, budget):
    i = _ce_inputs(R, D, V, True, R // 5)
    ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], i["weight"])
    for b in (budget, Bd.rnnt_ce_loss_workspace_bytes(Bd.RnntCeDesc(R, D, V, Bd.RNNT_BF16, -1, 0, bits, 0), True, budget)):
        _check_ce(_run_ce(i, True, budget=b, bits=bits), i, ref, True, bits)


@pytest.mark.parametrize("x_bf16", [True, False])
@pytest.mark.parametrize("b_bf16", [True, False])
@pytest.mark.parametrize("reduction", ["sum", "none"])
@pytest.mark.parametrize("R", [40, 150])
def test_cross_entropy_takes_a_bias_of_either_type(x_bf16, b_bf16, reduction, R):
    torch = _torch()
    from paper_2211_16270_amd import autograd as A
    i = _ce_inputs(R, 40, 130, x_bf16, 9)
    dt = torch.bfloat16 if x_bf16 else torch.float32
    b = _dev(i["b"], torch.bfloat16 if b_bf16 else torch.float32)
    i["b"] = _np(b)
    leaves = dict(dx=_dev(i["x"], dt), dW=_dev(i["W"], dt), db=b)
    for t in leaves.values():
        t.requires_grad_()
    w, lab = _dev(i["weight"], torch.float32), _dev(i["labels"], torch.int32)
    if reduction == "sum":
        loss = A.rnnt_ce_loss(*leaves.values(), lab, row_weight=w)
    else:
        loss = (A.rnnt_ce_loss(*leaves.values(), lab, reduction="none") * w).sum()
    (loss * 3.0).backward()
    ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], 3.0 * i["weight"])
    for k, t in leaves.items():
        assert t.grad.dtype == t.dtype, k
        # (1e-2: every bf16 gradient of the library; an fp32 one 1e-5, its bias' rounding to bf16 2^-8)
        tol = 1e-2 if x_bf16 else 2.0 ** -8 if t.dtype == torch.bfloat16 else 1e-5
        assert np.linalg.norm(_np(t.grad) - ref[k]) <= tol * np.linalg.norm(ref[k]), k


@pytest.mark.parametrize("R", [40, 300])
@pytest.mark.parametrize("together", [True, False])
def test_captured_forward_and_backward_passes(R, together):
    """In one graph, or a backward pass captured by itself: each of its replays gives the gradients of its forward pass' last one, however often it is replayed."""
    torch = _torch()
    from paper_2211_16270_amd import autograd as A
    D, V = 64, 200
    g = torch.Generator(device="cuda:0").manual_seed(R)
    n = lambda *s, k=1.0: (torch.randn(*s, generator=g, device="cuda:0") * k).bfloat16()
    x, W, b = n(R, D), n(D, V, k=D ** -0.5), n(V)
    lab = torch.randint(-1, V, (R,), generator=g, device="cuda:0", dtype=torch.int32)
    up = torch.tensor(4.0, device="cuda:0")                      # (a power of two: scaling rounds nothing)
    leaves = [t.requires_grad_() for t in (x, W, b)]
    # the code is loaded before the capture
    A.rnnt_ce_loss(*leaves, lab).backward()
    for t in leaves:
        t.grad = None
    torch.cuda.synchronize()
    pool = torch.cuda.graph_pool_handle()
    forward, backward = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(forward, pool=pool):
        loss = A.rnnt_ce_loss(*leaves, lab)
        if together:
            grads = torch.autograd.grad(loss, leaves, up)
    if not together:
        with torch.cuda.graph(backward, pool=pool):
            grads = torch.autograd.grad(loss, leaves, up)
    for k in range(3):
        with torch.no_grad():
            x.copy_(n(R, D))
        forward.replay()
        want = Bd.run_ce_fwd_bwd(x.detach(), W.detach(), b.detach(), lab, param_grads_bf16=3)
        for again in range(3):
            (forward if together else backward).replay()
            torch.cuda.synchronize()
            for got, key in zip(grads, ("dx", "dW", "db")):
                assert torch.equal(got, (want[key].float() * 4.0).bfloat16()), (k, again, key)
            torch.zeros(1 << 16, device="cuda:0").sum().item()


@pytest.mark.parametrize("R", [40, 2000])
def test_evaluation_computes_no_gradients(R):
    torch = _torch()
    from paper_2211_16270_amd import autograd as A
    D, V, N = 512, 8192, 1024
    i = _ce_inputs(R, D, V, True, R // 4)
    x, W, b = (_dev(i[k], torch.bfloat16).requires_grad_() for k in ("x", "W", "b"))
    w, lab = _dev(i["weight"], torch.float32), _dev(i["labels"], torch.int32)
    Wl = torch.full((D, N), 0.01, dtype=torch.bfloat16, device="cuda:0", requires_grad=True)

    def peak(f):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        r = f()
        torch.cuda.synchronize()
        return r, torch.cuda.max_memory_allocated() - before

    with torch.no_grad():
        loss, most = peak(lambda: A.rnnt_ce_loss(x, W, b, lab, row_weight=w))
        rows, _ = peak(lambda: A.rnnt_ce_loss(x, W, b, lab, reduction="none"))
        only, least = peak(lambda: Bd.run_ce_total(Bd.run_ce_fwd(x, W, b, lab)["loss"], w))
        y, kept = peak(lambda: A.rnnt_linear(x, Wl, None, "silu"))
        plain, bare = peak(lambda: Bd.run_linear_fwd(x, Wl, None, "silu")["y"])
    assert not loss.requires_grad and torch.equal(loss, only) and not y.requires_grad and torch.equal(y, plain)
    assert torch.equal(rows, Bd.run_ce_fwd(x, W, b, lab)["loss"])
    # neither dW nor the chunk of exponentials, nor the saved z
    assert most <= least and kept <= bare, (most, least, kept, bare)
    # with gradients the value is the same
    assert abs(float(A.rnnt_ce_loss(x, W, b, lab, row_weight=w)) - float(loss)) <= 1e-5 * abs(float(loss))


@pytest.mark.parametrize("M", [40, 400])
def test_tanh_of_small_arguments(M):
    """z = x W of one nonzero product each, exact in fp32; y is off by its rounding to bf16, 2^-8, and the function's 3.1e-5: below 2^-7 it is z, off by z^2 / 3
    (2.0e-5 of it), above 1 - 2 / (1 + e^{2z}) in fp32: the reciprocal of about 2 to 2^-23, doubled, the sum to 2^-24 and the exponential to 2^-23, times its
    slope of 1 / 2, are 2.4e-7 together."""
    torch = _torch()
    K, N = 64, 128
    g = np.random.default_rng(M)
    x, W = np.zeros((M, K)), np.zeros((K, N))
    x[:, 0] = np.exp(g.uniform(np.log(1e-12), np.log(2.0), M)) * g.choice([-1.0, 1.0], M)
    W[0] = np.exp(g.uniform(np.log(0.25), np.log(4.0), N)) * g.choice([-1.0, 1.0], N)
    xt, Wt = _dev(x, torch.bfloat16), _dev(W, torch.bfloat16)
    want = np.tanh(_np(xt) @ _np(Wt))
    got = _np(Bd.run_linear_fwd(xt, Wt, None, "tanh")["y"])
    over = np.abs(got - want) / np.abs(want)
    assert over.max() <= 2.0 ** -8 + 3.1e-5, over.max()
    assert bool((Bd.run_linear_fwd(torch.zeros_like(xt), Wt, None, "tanh")["y"] == 0).all())


def test_a_call_without_rows_leaves_the_state_it_took():
    torch = _torch()
    state = torch.tensor([123, 456], dtype=torch.int64, device="cuda:0")
    used, W = torch.zeros(2, dtype=torch.int64, device="cuda:0"), torch.zeros(8, 8, device="cuda:0")
    d = Bd.RnntLinearDesc(0, 8, 8, Bd.RNNT_F32, 0, 0.5, 0, 0, 0)
    assert Bd.rnnt_linear_fwd(d, None, W, None, None, state, used, None, None) == 0
    torch.cuda.synchronize()
    assert used.tolist() == [123, 456]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = Bd.run_linear_fwd(torch.zeros(0, 8, device="cuda:0"), W, None, dropout=0.5, rng_state=state, save=True, stream=side)
    side.synchronize()
    assert out["rng_used"].tolist() == [123, 456] and out["y"].shape == (0, 8)


@pytest.mark.parametrize("R,D,V", [(20, 512, 26624), (64, 704, 10624)])
def test_cross_entropy_of_few_rows_over_long_vocabularies(R, D, V):
    """Widths for which large tiles would be planned; operands in two values have small ones, and a plan for others is refused."""
    i = _ce_inputs(R, D, V, True, 3)
    ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], i["weight"])
    _check_ce(_run_ce(i, True, bits=3), i, ref, True, 3)


@pytest.mark.parametrize("M,K,N", [(1, 1088, 4032), (64, 1600, 2304)])
def test_linear_gradients_of_few_rows_and_wide_layers(M, K, N):
    i = _linear_inputs(M, K, N, True, res=False)
    ref = O.linear(i["x"], i["W"], i["b"], "silu", None, None, i["dy"])
    _check_linear(_run_linear(i, "silu", 0.0, True), i, ref, "silu", 0.0, True)
