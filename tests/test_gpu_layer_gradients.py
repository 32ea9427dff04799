"""How exact the layers' gradients are where a rounding to bfloat16 would show, and that no result depends on what a workspace held, on the GPU.

dW and db are asked for in fp32 here, so their only roundings are those of the score gradients or of dz inside.  Per entry those are off by
  cross entropy   the label's entry g = w (p - 1): half a step of (p - 1), 2^-9 w, as weights share one unit; with at most 64 rows 2^-17 |g|; the others, w p: an fp16
                  exponential, 2^-11, and one rounding, 2^-8 (at most 64 rows: 2^-16), of themselves;
  dz              dy act'(z) mask, 2^-8 of itself (at most 64 rows: 2^-16; nothing where act' is 0 or 1), and act' at a z rounded to fp16, 0.8 |z| 2^-11 |dy|,
and the sums and elementary functions add 2^-17 of the magnitudes at hand at these sizes (under 700 terms of 2^-24 each, 4e-6 relative)."""
import types

import numpy as np
import pytest

from paper_2211_16270_amd import binding as Bd
from tests import layer_oracle as O
from tests.test_gpu_layers import STATE, _ce_inputs, _dev, _linear_inputs, _np, _rounded, _run_ce, _run_linear

pytestmark = pytest.mark.gpu


def _ce_bounds(i, ref, few):
    """Bounds of |dh|'s errors"""
    real = i["labels"] != -1
    w = np.where(real, np.abs(i["weight"]).astype(np.float64), 0.0)
    err = (2.0 ** -11 + (2.0 ** -16 if few else 2.0 ** -8) + 2.0 ** -17) * np.abs(ref["dh"]) + w[:, None] * 2.0 ** -37
    r, y = np.nonzero(real)[0], i["labels"][real]
    err[r, y] = (2.0 ** -16 if few else 2.0 ** -9 + 2.0 ** -17) * (np.abs(ref["dh"][r, y]) if few else w[real])
    return err


def _check_params(got, i, ref, err, d):
    """err: bounds of the errors of ref[d], the gradient in front of the products"""
    x = np.abs(i["x"])
    mag = np.abs(ref[d])
    for k, b in (("dW", x.T @ (err + 2.0 ** -17 * mag)), ("db", (err + 2.0 ** -17 * mag).sum(0))):
        over = np.abs(got[k] - ref[k]) - b - 1e-30
        assert np.all(over <= 0), (k, over.max(), np.linalg.norm(got[k] - ref[k]) / np.linalg.norm(ref[k]))


@pytest.mark.parametrize("R", [7, 64, 90, 300])
@pytest.mark.parametrize("weight", [(1 + 2.0 ** -8) / 1024, 1.0 / 3, -(1 + 2.0 ** -8), 0.0])
def test_equal_weights_round_alike_but_little(R, weight):
    """The label's gradients of all rows lie near one value, which bfloat16 may have nothing near: here half a step away."""
    i = _ce_inputs(R, 64, 520, True, 0, seed=1, spread=0.5)
    i["b"] = i["b"] * 0.1
    i["weight"] = np.full(R, weight, dtype=np.float32)
    ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], i["weight"])
    _check_params(_run_ce(i, True), i, ref, _ce_bounds(i, ref, R <= 64), "dh")


@pytest.mark.parametrize("R", [7, 90])
@pytest.mark.parametrize("bf16", [True, False])
def test_gradients_of_rows_that_are_all_but_certain(R, bf16):
    """p near 1: the label's gradient w (p - 1) is a small number, not the difference of two rounded large ones."""
    D, V = 64, 300
    i = _ce_inputs(R, D, V, bf16, R // 5, seed=2, spread=0.1)
    # x's entry of its own label's row of W: scores of about 14 there, 0 elsewhere
    i["labels"] = np.where(i["labels"] < 0, -1, np.arange(R) % D).astype(np.int32)
    i["x"] = _rounded(i["x"] * 0.05, bf16)
    i["x"][np.arange(R), np.arange(R) % D] = 4.0
    i["W"][np.arange(D), np.arange(D)] = 3.5
    i["b"] = i["b"] * 0.1
    ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], i["weight"])
    real = i["labels"] >= 0
    q = -ref["dh"][np.nonzero(real)[0], i["labels"][real]] / i["weight"][real]
    assert 1e-5 < q.min() and q.max() < 1e-2
    got = _run_ce(i, bf16)
    # scores of about 14, sums of 64 products: off by 64 2^-24 14 at most, 2^-14, and q = 1 - p by as much of itself.  The sum of the exponentials is 1 + q, and each
    # addition that it goes through rounds it by 2^-24: at most 31 within a lane's columns of a tile, 2 between lanes, 1 between waves, 5 to 9 between tiles (300
    # columns in parts of 64 or 32), and one more in the logarithm: 40 2^-24, absolutely
    few = R <= 64
    err = _ce_bounds(i, ref, few) if bf16 else 8 * 2.0 ** -24 * np.abs(ref["dh"])
    r, y = np.nonzero(real)[0], i["labels"][real]
    err += 2.0 ** -13 * np.abs(ref["dh"])
    w = np.abs(i["weight"][real]).astype(np.float64)
    # (bf16 rounds p - 1 itself, relatively: not by 2^-9 of the weight, as a difference could be, but by 2^-8 of itself)
    err[r, y] = (2.0 ** -8 if bf16 and not few else 2.0 ** -16) * np.abs(ref["dh"][r, y]) + w * (2.0 ** -13 * q + 40 * 2.0 ** -24)
    _check_params(got, i, ref, err, "dh")


@pytest.mark.parametrize("name,p,M", [("none", 0.1, 200), ("relu", 0.3, 200), ("relu", 0.0, 70), ("none", 0.4, 9), ("silu", 0.1, 300), ("gelu", 0.3, 64),
                                      ("tanh", 0.0, 1), ("silu", 0.3, 33), ("gelu", 0.0, 65)])
@pytest.mark.parametrize("K,N", [(64, 128), (72, 130), (33, 100)])
def test_dz_is_rounded_once_or_not_at_all(name, p, M, K, N):
    i = _linear_inputs(M, K, N, True, res=False, seed=3)
    ref = O.linear(i["x"], i["W"], i["b"], name, None, O.keep_scale(M, N, *STATE, p), i["dy"])
    got = _run_linear(i, name, p, True)
    scale = 1.0 / (1.0 - p) * 1.001
    zerr = (K + 16) * 2.0 ** -23 * (np.abs(i["x"]) @ np.abs(i["W"]) + 1.0)
    if name in ("none", "relu"):
        err = np.zeros((M, N))
        if name == "relu":
            err = np.where(np.abs(ref["z"]) <= zerr, np.abs(i["dy"]) * scale, 0.0)
    else:
        err = (2.0 ** -16 if M <= 64 else 2.0 ** -8) * np.abs(ref["dz"]) + 0.8 * np.abs(i["dy"]) * scale * (2.0 ** -11 * np.abs(ref["z"]) + zerr + 5e-6)
    _check_params(got, i, ref, err, "dz")
    if M <= 64:
        # dx is rounded itself; in front of that its error is the rest's alone
        aw = np.abs(i["W"])
        b = (err + 2.0 ** -17 * np.abs(ref["dz"])) @ aw.T + 2.0 ** -8 * 1.01 * np.abs(ref["dx"]) + 1e-30
        assert np.all(np.abs(got["dx"] - ref["dx"]) <= b)


def test_infinite_gradients_of_a_few_rows_leave_no_nan():
    torch = _torch()
    i = _linear_inputs(5, 64, 72, True, res=False, seed=4)
    x, W, dy = (_dev(i[k], torch.bfloat16) for k in ("x", "W", "dy"))
    x, W, dy = x.abs() + 1, W.abs() + 2 ** -6, dy.abs() + 1
    dy[2, 5] = float("inf")
    b = torch.full((72,), 40.0, device="cuda:0")                 # (act' = 1)
    f = Bd.run_linear_fwd(x, W, b, "silu", save=True)
    g = Bd.run_linear_bwd(x, W, dy, "silu", f["saved"])
    assert bool(torch.isinf(g["dx"][2].float()).all()) and bool(torch.isfinite(g["dx"][[0, 1, 3, 4]].float()).all())
    assert bool(torch.isinf(g["dW"][:, 5]).all()) and bool(torch.isinf(g["db"][5])) and int(torch.isfinite(g["dW"]).sum()) == 64 * 71


def _torch():
    import torch
    return torch


def _poisoned(nbytes, kind):
    torch = _torch()
    n = max(1024, nbytes)
    if kind == "zero":
        return types.SimpleNamespace(buf=torch.zeros(n, dtype=torch.uint8, device="cuda:0"))
    # fp32 of 1e9 everywhere (bf16 and fp16: 1e9 and a large one), or NaN of every type
    word = np.float32(1e9).view(np.int32).item() if kind == "large" else -1
    return types.SimpleNamespace(buf=torch.full(((n + 3) // 4,), word, dtype=torch.int32, device="cuda:0").view(torch.uint8)[:n])


@pytest.mark.parametrize("M,K,N,act,p", [(1, 64, 710, "silu", 0.1), (11, 64, 710, "gelu", 0.0), (40, 2600, 33, "none", 0.0), (64, 63, 65, "tanh", 0.0),
                                         (70, 63, 65, "relu", 0.1), (130, 72, 96, "none", 0.0), (200, 2048, 129, "silu", 0.0)])
@pytest.mark.parametrize("bf16", [True, False])
def test_a_linear_layer_reads_nothing_of_its_workspace_that_it_did_not_write(M, K, N, act, p, bf16):
    torch = _torch()
    dt = torch.bfloat16 if bf16 else torch.float32
    i = _linear_inputs(M, K, N, bf16, res=True, seed=6)
    x, W, b, res, dy = _dev(i["x"], dt), _dev(i["W"], dt), _dev(i["b"], torch.float32), _dev(i["residual"], dt), _dev(i["dy"], dt)
    rng = torch.tensor(STATE, dtype=torch.int64, device="cuda:0")
    desc = Bd.RnntLinearDesc(M, K, N, int(bf16), Bd.ACTIVATIONS.index(act), p, 0, 0, 0)
    sizes = [Bd.rnnt_linear_workspace_bytes(desc, back) for back in (False, True)]
    results = {}
    for kind in ("zero", "large", "nan"):
        f = Bd.run_linear_fwd(x, W, b, act, res, p, rng, save=True, workspace=_poisoned(sizes[0], kind))
        g = Bd.run_linear_bwd(x, W, dy, act, f["saved"], p, rng, workspace=_poisoned(sizes[1], kind))
        results[kind] = [f["y"], g["dx"], g["dW"], g["db"]]
    for kind in ("large", "nan"):
        for u, v in zip(results["zero"], results[kind]):
            assert torch.equal(u, v), kind


@pytest.mark.parametrize("R,D,V,pad", [(1, 64, 710, 0), (11, 64, 710, 1), (64, 63, 65, 9), (33, 128, 96, 33), (90, 70, 130, 50), (300, 64, 4100, 280),
                                       (17000, 8, 40, 16990), (70001, 8, 24, 30000)])
@pytest.mark.parametrize("bf16", [True, False])
def test_the_cross_entropy_reads_nothing_of_its_workspace_that_it_did_not_write(R, D, V, pad, bf16):
    torch = _torch()
    dt = torch.bfloat16 if bf16 else torch.float32
    i = _ce_inputs(R, D, V, bf16, pad, seed=7)
    x, W, b, lab, w = (_dev(i["x"], dt), _dev(i["W"], dt), _dev(i["b"], torch.float32), _dev(i["labels"], torch.int32), _dev(i["weight"], torch.float32))
    desc = Bd.RnntCeDesc(R, D, V, int(bf16), -1, 0, 0, 0)
    sizes = [Bd.rnnt_ce_loss_workspace_bytes(desc, grads) for grads in (False, True)]
    results = {}
    for kind in ("zero", "large", "nan"):
        f = Bd.run_ce_fwd(x, W, b, lab, workspace=_poisoned(sizes[0], kind))
        g = Bd.run_ce_fwd_bwd(x, W, b, lab, w, workspace=_poisoned(sizes[1], kind))
        results[kind] = [f["loss"], g["loss"], g["dx"], g["dW"], g["db"]]
    for kind in ("large", "nan"):
        for u, v in zip(results["zero"], results[kind]):
            assert torch.equal(u, v), kind
    ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], i["weight"])
    assert np.all(np.abs(_np(results["nan"][0]) - ref["loss"]) <= 2e-5 * (1 + np.abs(ref["loss"])))


def test_a_captured_backward_pass_of_an_eager_forward_call_scales_once():
    torch = _torch()
    from paper_2211_16270_amd import autograd as A
    i = _ce_inputs(90, 64, 128, True, 9, seed=8)
    lab = _dev(i["labels"], torch.int32)
    g = torch.full((), 0.25, device="cuda:0")

    def leaves():
        return [_dev(i[k], torch.bfloat16).requires_grad_() for k in ("x", "W")]

    x, W = leaves()
    ref = torch.autograd.grad(A.rnnt_ce_loss(x, W, None, lab), (x, W), g)
    x, W = leaves()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        loss = A.rnnt_ce_loss(x, W, None, lab)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = torch.autograd.grad(loss, (x, W), g)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(got, ref):
            assert torch.equal(u, v)


@pytest.mark.parametrize("name", Bd.ACTIVATIONS)
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("M", [40, 150])
def test_dropped_entries_take_nothing_from_an_infinite_gradient(name, bf16, M):
    torch = _torch()
    K, N = 64, 72
    i = _linear_inputs(M, K, N, bf16, res=False, seed=9)
    dt = torch.bfloat16 if bf16 else torch.float32
    x, W, b, dy = _dev(i["x"], dt), _dev(i["W"], dt), _dev(i["b"], torch.float32), _dev(i["dy"], dt)
    rng = torch.tensor(STATE, dtype=torch.int64, device="cuda:0")
    dropped = torch.from_numpy(O.keep_scale(M, N, *STATE, 0.3) == 0).cuda()
    f = Bd.run_linear_fwd(x, W, b, name, None, 0.3, rng, save=True)
    zero, wild = dy.masked_fill(dropped, 0.0), dy.masked_fill(dropped, float("inf"))
    wild[0][dropped[0]] = float("nan")
    g, h = (Bd.run_linear_bwd(x, W, d, name, f["saved"], 0.3, rng) for d in (zero, wild))
    for k in ("dx", "dW", "db"):
        assert torch.equal(g[k], h[k]), k
    # and an infinite z that is dropped, or kept where act' is 0 or 1 there
    big = torch.full((N,), 1e30, device="cuda:0")
    for sign in (1.0, -1.0):
        f = Bd.run_linear_fwd(x, W, sign * big, name, None, 0.3, rng, save=True)
        g = Bd.run_linear_bwd(x, W, dy, name, f["saved"], 0.3, rng)
        slope = {"none": 1.0, "tanh": 0.0}.get(name, 1.0 if sign > 0 else 0.0)
        ref = (dy.double() * (~dropped) * (65536.0 / (65536 - round(0.3 * 65536))) * slope).sum(0)
        assert torch.allclose(g["db"].double(), ref, rtol=1e-5, atol=1e-4), (sign, name)
