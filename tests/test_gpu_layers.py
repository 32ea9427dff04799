"""The layers beside the transducer loss on the GPU, against the 64-bit oracle of layer_oracle.py.

Tolerances.  A rounding to bfloat16 is off by at most 2^-8 of the value, to fp16 2^-11, to fp32 2^-24.  With RNNT_BF16 (products of bfloat16 values are exact in
fp32, sums of n of them off by at most n 2^-24 of the sum of their magnitudes):
  y       one rounding, plus (K + 16) 2^-24 of |x| |W| + |b|, times the activation's largest slope (1.13) and the dropout's scale, plus the
          elementary functions' 4e-6 of the magnitude at hand;
  dz      two relative errors: its own rounding, 2^-8, and act' at a z rounded to fp16, |z| 2^-11 times the largest |act''| (0.8); its sums carry them through |W|, |x|;
  dh      weight * probability out of an fp16 exponential (2^-11, or 2^-39 of the part's largest) rounded to bf16: 2^-8 + 2^-10 of its entries' magnitudes.
A gradient is compared entry by entry with the bound that these give, and as a whole: 1e-2 of its norm, which is what every gradient of this library is
held to."""
import numpy as np
import pytest

from paper_2211_16270_amd import binding as Bd
from tests import layer_oracle as O

pytestmark = pytest.mark.gpu

U8, U11, U24 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24
STATE = (0x123456789ABCDEF, 0x0FEDCBA987654321)


def _torch():
    import torch
    return torch


def _dev(a, dtype):
    torch = _torch()
    return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda:0", dtype=dtype)


def _rounded(a, bf16):
    torch = _torch()
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64))
    return t.to(torch.bfloat16 if bf16 else torch.float32).double().numpy()


def _np(t):
    return t.detach().double().cpu().numpy()


def _linear_inputs(M, K, N, bf16, res, seed=0):
    g = np.random.default_rng(seed * 1000 + M * 7 + K * 3 + N)
    r = lambda *s: _rounded(g.normal(size=s), bf16)
    return dict(x=r(M, K), W=_rounded(g.normal(size=(K, N)) / np.sqrt(K), bf16), b=g.normal(size=N).astype(np.float32).astype(np.float64) * 0.25,
                residual=r(M, N) if res else None, dy=r(M, N))


def _run_linear(i, name, p, bf16, want=("dx", "dW", "db"), bits=0):
    torch = _torch()
    dt = torch.bfloat16 if bf16 else torch.float32
    x, W, dy = (_dev(i[k], dt) for k in ("x", "W", "dy"))
    b = None if i["b"] is None else _dev(i["b"], torch.float32)
    res = None if i["residual"] is None else _dev(i["residual"], dt)
    rng = torch.tensor(STATE, dtype=torch.int64, device="cuda:0") if p else None
    f = Bd.run_linear_fwd(x, W, b, name, res, p, rng, save=True)
    g = Bd.run_linear_bwd(x, W, dy, name, f["saved"], p, f["rng_used"], param_grads_bf16=bits, want=want)
    torch.cuda.synchronize()
    if p:
        assert f["rng_used"].tolist() == list(STATE)
    return {k: None if v is None else _np(v) for k, v in dict(y=f["y"], **g).items()}


def _check_linear(got, i, ref, name, p, bf16, bits=0):
    u = U8 if bf16 else U24
    M, K = i["x"].shape
    N = i["W"].shape[1]
    ax, aw, ady = np.abs(i["x"]), np.abs(i["W"]), np.abs(ref["dz"])
    scale = 1.0 / (1.0 - p) * 1.001
    # (the fp32 path's products: six of three parts, 2^-24 of each at most, like a rounded product)
    zerr = (K + 16) * 2 * U24 * (ax @ aw + 1.0)
    yb = u * np.abs(ref["y"]) * 1.01 + scale * (1.13 * zerr + 4e-6 * (np.abs(ref["z"]) + 1e-3)) + 4 * U24 * np.abs(ref["y"])
    assert np.all(np.abs(got["y"] - ref["y"]) <= yb), "y"
    slope = 0.8 * np.abs(i["dy"]) * scale * ((U11 * 1.01 if bf16 else U24) * np.abs(ref["z"]) + zerr + 1e-7 + 4e-6) if name != "none" else 0.0
    if name == "relu":
        # a z within its error of zero may fall on either side
        slope = np.where(np.abs(ref["z"]) <= zerr, np.abs(i["dy"]) * scale, 0.0)
    own = 2.0 ** -8 * 1.01 if bf16 else 4 * U24
    dzb = own * ady + slope
    for k, b in (("dx", dzb @ aw.T + (N + 16) * 2 * U24 * (ady @ aw.T)), ("dW", ax.T @ dzb + (M + 16) * 2 * U24 * (ax.T @ ady)),
                 ("db", (slope + 4 * U24 * ady).sum(0) + (M + 16) * U24 * ady.sum(0) if name != "none" else (M + 16) * U24 * ady.sum(0))):
        if got[k] is None:
            continue
        rounded16 = (k == "dx" and bf16) or (k == "dW" and bits & 1) or (k == "db" and bits & 2)
        b = b + (U8 if rounded16 else U24) * 1.01 * np.abs(ref[k]) + 1e-30
        assert np.all(np.abs(got[k] - ref[k]) <= b), (k, np.max(np.abs(got[k] - ref[k]) / b))
        if M * N >= 64:
            n = np.linalg.norm(ref[k])
            assert np.linalg.norm(got[k] - ref[k]) <= (1e-2 if bf16 else 1e-5) * n + 1e-30, k


# one row and many, sizes that are multiples of nothing, of the tiles, one beyond them; the few-rows kernel's limits (16, 32, 64), a long sum in it, split sums
LINEAR_SIZES = [(1, 1, 1), (1, 640, 2560), (2, 7, 9), (16, 64, 64), (17, 33, 31), (33, 2600, 40), (64, 129, 257), (65, 64, 8), (100, 63, 65), (128, 128, 128),
                (129, 320, 130), (255, 72, 256), (257, 64, 513), (300, 2048, 72), (1000, 16, 24)]


@pytest.mark.parametrize("M,K,N", LINEAR_SIZES)
@pytest.mark.parametrize("bf16", [True, False])
def test_linear_sizes(M, K, N, bf16):
    n = LINEAR_SIZES.index((M, K, N))
    name, p = Bd.ACTIVATIONS[n % 5], (0.0, 0.25, 0.1)[n % 3]
    i = _linear_inputs(M, K, N, bf16, res=n % 2 == 0)
    ref = O.linear(i["x"], i["W"], i["b"], name, i["residual"], O.keep_scale(M, N, *STATE, p), i["dy"])
    bits = (3 if n % 2 else 0) if bf16 else 0
    _check_linear(_run_linear(i, name, p, bf16, bits=bits), i, ref, name, p, bf16, bits)


@pytest.mark.parametrize("name", Bd.ACTIVATIONS)
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("p", [0.0, 0.4])
def test_linear_activations(name, bf16, p):
    M, K, N = 200, 96, 120
    i = _linear_inputs(M, K, N, bf16, res=True, seed=5)
    i["x"] = _rounded(i["x"] * np.linspace(0.1, 6.0, M)[:, None], bf16)         # small and large arguments
    ref = O.linear(i["x"], i["W"], i["b"], name, i["residual"], O.keep_scale(M, N, *STATE, p), i["dy"])
    _check_linear(_run_linear(i, name, p, bf16), i, ref, name, p, bf16)


@pytest.mark.parametrize("M,N,K,bf16", [(3, 41, 8, True), (70, 41, 64, True), (130, 264, 64, True), (300, 24, 4096, True), (40, 43, 8, False)])
def test_dropout_masks_are_the_published_generators(M, N, K, bf16):
    """x = 0, b = 1: the output is the mask itself."""
    torch = _torch()
    dt = torch.bfloat16 if bf16 else torch.float32
    x, W, b = torch.zeros(M, K, dtype=dt, device="cuda:0"), torch.zeros(K, N, dtype=dt, device="cuda:0"), torch.ones(N, device="cuda:0")
    for p, state in ((0.1, (0, 0)), (0.5, STATE), (0.9, (2 ** 62 + 5, 7))):
        rng = torch.tensor(state, dtype=torch.int64, device="cuda:0")
        y = _np(Bd.run_linear_fwd(x, W, b, "none", None, p, rng)["y"])
        ref = _rounded(O.keep_scale(M, N, *state, p), bf16)
        np.testing.assert_array_equal(y, ref)


def test_bias_of_either_type_or_none():
    torch = _torch()
    i = _linear_inputs(150, 64, 70, True, res=False)
    i["b"] = _rounded(i["b"], True)
    x, W = _dev(i["x"], torch.bfloat16), _dev(i["W"], torch.bfloat16)
    y32 = Bd.run_linear_fwd(x, W, _dev(i["b"], torch.float32))["y"]
    y16 = Bd.run_linear_fwd(x, W, _dev(i["b"], torch.bfloat16))["y"]
    assert torch.equal(y32, y16)
    none, zero = Bd.run_linear_fwd(x, W)["y"], Bd.run_linear_fwd(x, W, torch.zeros(70, device="cuda:0"))["y"]
    assert torch.equal(none, zero)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("name", ["none", "silu"])
def test_linear_accumulates_parameter_gradients_and_leaves_out_what_is_not_wanted(bf16, name):
    torch = _torch()
    M, K, N = 130, 72, 66
    i = _linear_inputs(M, K, N, bf16, res=False)
    ref = O.linear(i["x"], i["W"], i["b"], name, None, None, i["dy"])
    dt = torch.bfloat16 if bf16 else torch.float32
    x, W, dy, b = _dev(i["x"], dt), _dev(i["W"], dt), _dev(i["dy"], dt), _dev(i["b"], torch.float32)
    saved = Bd.run_linear_fwd(x, W, b, name, save=True)["saved"]
    dW, db = torch.full((K, N), 3.0, device="cuda:0"), torch.full((N,), -2.0, device="cuda:0")
    Bd.run_linear_bwd(x, W, dy, name, saved, accumulate_into=(dW, db))
    plain = Bd.run_linear_bwd(x, W, dy, name, saved)
    # (an fp32 addition of the same sums: off by half a step of the result)
    np.testing.assert_allclose(_np(dW), _np(plain["dW"]) + 3.0, atol=1e-6 * (3 + np.abs(ref["dW"]).max()), rtol=0)
    np.testing.assert_allclose(_np(db), _np(plain["db"]) - 2.0, atol=1e-6 * (2 + np.abs(ref["db"]).max()), rtol=0)
    for want in (("dx",), ("dW",), ("db",), ("dx", "db")):
        g = Bd.run_linear_bwd(x, W, dy, name, saved, want=want)
        for k in ("dx", "dW", "db"):
            assert (g[k] is None) == (k not in want)
            if k in want:
                assert np.linalg.norm(_np(g[k]) - ref[k]) <= (1e-2 if bf16 else 1e-5) * np.linalg.norm(ref[k])


@pytest.mark.parametrize("bf16", [True, False])
def test_no_rows_at_all(bf16):
    torch = _torch()
    dt = torch.bfloat16 if bf16 else torch.float32
    x, W = torch.zeros(0, 24, dtype=dt, device="cuda:0"), torch.ones(24, 40, dtype=dt, device="cuda:0")
    f = Bd.run_linear_fwd(x, W, None, "silu", save=True)
    assert f["y"].shape == (0, 40)
    g = Bd.run_linear_bwd(x, W, f["y"], "silu", f["saved"])
    assert g["dx"].shape == (0, 24) and float(g["dW"].abs().sum()) == 0 and float(g["db"].abs().sum()) == 0
    dW, db = torch.full((24, 40), 2.0, device="cuda:0"), torch.full((40,), 2.0, device="cuda:0")
    Bd.run_linear_bwd(x, W, f["y"], "silu", f["saved"], accumulate_into=(dW, db))
    assert float((dW - 2).abs().sum()) == 0 and float((db - 2).abs().sum()) == 0
    lab = torch.zeros(0, dtype=torch.int32, device="cuda:0")
    assert Bd.run_ce_fwd(x, W, None, lab)["loss"].shape == (0,)
    o = Bd.run_ce_fwd_bwd(x, W, None, lab)
    assert o["dx"].shape == (0, 24) and float(o["dW"].abs().sum()) == 0 and float(o["db"].abs().sum()) == 0
    Bd.run_ce_fwd_bwd(x, W, None, lab, accumulate_into=(dW, db))
    assert float((dW - 2).abs().sum()) == 0 and float((db - 2).abs().sum()) == 0
    assert float(Bd.run_ce_total(o["loss"])) == 0.0


@pytest.mark.parametrize("M", [5, 200])
def test_rows_do_not_touch_each_other(M):
    """Infinities and NaN in one row stay there; the limits of the activations at infinity."""
    torch = _torch()
    K, N = 64, 96
    i = _linear_inputs(M, K, N, True, res=False)
    x, W, b = _dev(i["x"], torch.bfloat16), _dev(np.abs(i["W"]) + 2 ** -6, torch.bfloat16), _dev(i["b"], torch.float32)
    clean = {n: Bd.run_linear_fwd(x, W, b, n)["y"] for n in Bd.ACTIVATIONS}
    x[1, 3], x[2, 5], x[M - 1, 0] = float("inf"), -float("inf"), float("nan")
    limits = dict(none=(np.inf, -np.inf), relu=(np.inf, 0.0), silu=(np.inf, 0.0), gelu=(np.inf, 0.0), tanh=(1.0, -1.0))
    rest = [r for r in range(M) if r not in (1, 2, M - 1)]
    for n in Bd.ACTIVATIONS:
        y = Bd.run_linear_fwd(x, W, b, n)["y"]
        assert torch.equal(y[rest], clean[n][rest]), n
        assert bool((y[1].float() == limits[n][0]).all()) and bool((y[2].float() == limits[n][1]).all()), n
        assert bool(torch.isnan(y[M - 1].float()).all()), n


def test_outputs_and_workspace_keep_to_their_bounds():
    torch = _torch()
    for M, K, N in ((70, 63, 65), (64, 2560, 24), (200, 72, 40)):
        i = _linear_inputs(M, K, N, True, res=False)
        x, W, dy = (_dev(i[k], torch.bfloat16) for k in ("x", "W", "dy"))
        guard = 256

        def fenced(shape, dtype):
            n = int(np.prod(shape))
            buf = torch.full((guard + n + guard,), 7.0, device="cuda:0").to(dtype)
            return buf, buf[guard:guard + n].view(shape)

        def intact(buf):
            assert bool((buf[:guard] == 7).all()) and bool((buf[-guard:] == 7).all())

        desc = Bd.RnntLinearDesc(M, K, N, 1, 2, 0.25, 0, 0, 0)
        rng = torch.tensor(STATE, dtype=torch.int64, device="cuda:0")
        yb, y = fenced((M, N), torch.bfloat16)
        sb, saved = fenced((M, N), torch.float16)
        nbytes = [Bd.rnnt_linear_workspace_bytes(desc, w) for w in (False, True)]
        ws = [torch.full((n + 1024,), 91, dtype=torch.uint8, device="cuda:0") for n in nbytes]
        assert Bd.rnnt_linear_fwd(desc, x, W, None, None, rng, None, y, saved, ws[0][:nbytes[0]]) == 0
        xb, dx = fenced((M, K), torch.bfloat16)
        wb, dW = fenced((K, N), torch.float32)
        bb, db = fenced((N,), torch.float32)
        assert Bd.rnnt_linear_bwd(desc, x, W, saved, rng, dy, dx, dW, db, ws[1][:nbytes[1]]) == 0
        torch.cuda.synchronize()
        for buf in (yb, sb, xb, wb, bb):
            intact(buf)
        for w, n in zip(ws, nbytes):
            assert bool((w[n:] == 91).all())
        lab = torch.zeros(M, dtype=torch.int32, device="cuda:0")
        lab[::3] = -1
        cd = Bd.RnntCeDesc(M, K, N, 1, -1, 0, 3, 0)
        n = Bd.rnnt_ce_loss_workspace_bytes(cd, True)
        ws = torch.full((n + 1024,), 91, dtype=torch.uint8, device="cuda:0")
        (lb, loss), (xb, dx), (wb, dW), (bb, db) = (fenced((M,), torch.float32), fenced((M, K), torch.bfloat16), fenced((K, N), torch.bfloat16),
                                                    fenced((N,), torch.bfloat16))
        assert Bd.rnnt_ce_loss_fwd_bwd(cd, x, W, None, lab, None, loss, dx, dW, db, ws[:n]) == 0
        torch.cuda.synchronize()
        for buf in (lb, xb, wb, bb):
            intact(buf)
        assert bool((ws[n:] == 91).all())


def test_more_than_2_to_the_32_outputs():
    torch = _torch()
    M, K, N = 1050000, 8, 4104
    assert M * N > 2 ** 32
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda:0")
    x[:, 0] = (torch.arange(M, device="cuda:0") % 251).bfloat16()
    W = torch.zeros(K, N, dtype=torch.bfloat16, device="cuda:0")
    W[0] = (torch.arange(N, device="cuda:0") % 127 - 63).bfloat16()
    y = Bd.run_linear_fwd(x, W)["y"]
    torch.cuda.synchronize()
    for r in (0, 1, M // 2, M - 300, M - 1):
        ref = (float(r % 251) * W[0].float()).bfloat16()
        assert torch.equal(y[r], ref), r
    del y, x
    torch.cuda.empty_cache()


# ---- cross entropy ---------------------------------------------------------------------------------------------------------------------

def _ce_inputs(R, D, V, bf16, pad, seed=0, spread=2.0):
    g = np.random.default_rng(seed * 1000 + R * 5 + D * 3 + V)
    lab = g.integers(0, V, size=R).astype(np.int32)
    lab[g.permutation(R)[:pad]] = -1
    return dict(x=_rounded(g.normal(size=(R, D)), bf16), W=_rounded(g.normal(size=(D, V)) * spread / np.sqrt(D), bf16),
                b=(g.normal(size=V) * 0.5).astype(np.float32).astype(np.float64), labels=lab, weight=g.uniform(0.2, 2.0, size=R).astype(np.float32))


def _run_ce(i, bf16, budget=0, weight=True, bits=0, **kw):
    torch = _torch()
    dt = torch.bfloat16 if bf16 else torch.float32
    o = Bd.run_ce_fwd_bwd(_dev(i["x"], dt), _dev(i["W"], dt), None if i["b"] is None else _dev(i["b"], torch.float32), _dev(i["labels"], torch.int32),
                          _dev(i["weight"], torch.float32) if weight else None, budget_bytes=budget, param_grads_bf16=bits, **kw)
    torch.cuda.synchronize()
    return {k: None if v is None else _np(v) for k, v in o.items()}


def _check_ce(got, i, ref, bf16, bits=0):
    real = i["labels"] != -1
    D, V = i["W"].shape
    x = np.where(real[:, None], i["x"], 0.0)
    herr = (D + 16) * 2 * U24 * (np.abs(x) @ np.abs(i["W"]) + 1.0).max(1)
    fin = np.isfinite(ref["loss"])
    np.testing.assert_array_equal(got["loss"][~fin], ref["loss"][~fin])
    lb = 2 * herr + 2e-6 * (np.abs(ref["loss"]) + np.abs(np.where(np.isfinite(ref["h"]), ref["h"], 0)).max(1) + 1.0)
    assert np.all(np.abs(got["loss"] - ref["loss"])[fin] <= lb[fin]), "loss"
    assert np.all(got["loss"][~real] == 0) and np.all(got["dx"][~real] == 0)
    own = (2.0 ** -8 + 2.0 ** -10) if bf16 else 1e-5
    w = np.abs(i["weight"]) * real if i["weight"] is not None else real * 1.0
    dhb = own * np.abs(ref["dh"]) + w[:, None] * 2.0 ** -37 + 2 * herr[:, None] * np.abs(ref["dh"])
    # (the label's entry: weight (p - 1), each of the two with its error)
    known = real & (i["labels"] >= 0) & (i["labels"] < V)
    dhb[np.arange(len(real))[known], i["labels"][known]] += own * w[known]
    aw, ax = np.abs(i["W"]), np.abs(x)
    for k, b in (("dx", dhb @ aw.T), ("dW", ax.T @ dhb), ("db", dhb.sum(0))):
        if got[k] is None:
            continue
        rounded16 = (k == "dx" and bf16) or (k == "dW" and bits & 1) or (k == "db" and bits & 2)
        mag = dict(dx=np.abs(ref["dh"]) @ aw.T, dW=ax.T @ np.abs(ref["dh"]), db=np.abs(ref["dh"]).sum(0))[k]
        b = b + (U8 if rounded16 else U24) * 1.01 * np.abs(ref[k]) + (max(V, len(real)) + 16) * 2 * U24 * mag + 1e-30
        assert np.all(np.abs(got[k] - ref[k]) <= b), (k, np.nanmax(np.abs(got[k] - ref[k]) / b))
        n = np.linalg.norm(ref[k])
        assert np.linalg.norm(got[k] - ref[k]) <= (1e-2 if bf16 else 1e-5) * n + 1e-30, k


CE_SIZES = [(1, 1, 2, 0), (1, 64, 64, 0), (3, 70, 130, 1), (16, 33, 31, 3), (40, 70, 130, 7), (64, 128, 700, 20), (65, 64, 300, 30), (100, 63, 65, 0),
            (129, 320, 1000, 60), (256, 128, 256, 0), (257, 72, 513, 256), (300, 64, 4100, 100), (700, 192, 96, 650)]


@pytest.mark.parametrize("R,D,V,pad", CE_SIZES)
@pytest.mark.parametrize("bf16", [True, False])
def test_cross_entropy_sizes(R, D, V, pad, bf16):
    i = _ce_inputs(R, D, V, bf16, pad)
    ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], i["weight"])
    bits = 3 if bf16 and CE_SIZES.index((R, D, V, pad)) % 2 else 0
    _check_ce(_run_ce(i, bf16, bits=bits), i, ref, bf16, bits)
    torch = _torch()
    dt = torch.bfloat16 if bf16 else torch.float32
    loss = _np(Bd.run_ce_fwd(_dev(i["x"], dt), _dev(i["W"], dt), _dev(i["b"], torch.float32), _dev(i["labels"], torch.int32))["loss"])
    got = dict(loss=loss, dx=np.zeros_like(ref["dx"]), dW=None, db=None)
    fin = np.isfinite(ref["loss"])
    assert np.all(np.abs(loss - ref["loss"])[fin] <= 1e-5 * (np.abs(ref["loss"])[fin] + 1)) and got["dW"] is None


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("R,pad", [(3000, 1200), (20000, 9000)])
def test_cross_entropy_in_chunks_and_of_many_rows(bf16, R, pad):
    """Several chunks of rows, the last ones empty; more rows than one workgroup counts itself."""
    i = _ce_inputs(R, 40, 300, bf16, pad)
    ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], i["weight"])
    whole = _run_ce(i, bf16)
    _check_ce(whole, i, ref, bf16)
    d = Bd.RnntCeDesc(R, 40, 300, int(bf16), -1, 0, 0, 0)
    smallest = Bd.rnnt_ce_loss_workspace_bytes(d, True, 1)
    assert smallest < Bd.rnnt_ce_loss_workspace_bytes(d, True)
    for budget in (1, smallest + (1 << 20)):
        for bits in ((0, 3) if bf16 else (0,)):
            _check_ce(_run_ce(i, bf16, budget=budget, bits=bits), i, ref, bf16, bits)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("R", [20, 200])
def test_cross_entropy_padding_may_hold_anything(bf16, R):
    i = _ce_inputs(R, 64, 96, bf16, R // 3)
    clean = _run_ce(i, bf16)
    dirty = dict(i, x=i["x"].copy())
    dirty["x"][i["labels"] == -1] = np.nan
    got = _run_ce(dirty, bf16)
    for k in ("loss", "dx", "dW", "db"):
        np.testing.assert_array_equal(got[k], clean[k])
    i["labels"][:] = -1
    got = _run_ce(dict(dirty, labels=i["labels"]), bf16)
    for k in ("loss", "dx", "dW", "db"):
        assert np.all(got[k] == 0), k


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("R", [9, 150])
def test_cross_entropy_of_masked_vocabularies_and_labels_outside(bf16, R):
    V = 200
    i = _ce_inputs(R, 64, V, bf16, 2)
    i["b"][50:] = -np.inf                                     # out of the vocabulary, a whole part of it among them
    i["b"][10] = -3.4028234663852886e38                       # the type's lowest value
    lab = np.where(i["labels"] >= 0, i["labels"] % 50, -1).astype(np.int32)
    lab[0], lab[1], lab[2], lab[3], lab[4] = 3, 120, V, 2 ** 31 - 1, -7
    i["labels"] = lab
    ref = O.cross_entropy(i["x"], i["W"], i["b"], lab, i["weight"])
    assert np.isinf(ref["loss"][[1, 2, 3, 4]]).all()
    _check_ce(_run_ce(i, bf16), i, ref, bf16)
    # no entry possible at all: the label's part of the gradient alone
    i["b"][:] = -np.inf
    ref = O.cross_entropy(i["x"], i["W"], i["b"], lab, i["weight"])
    got = _run_ce(i, bf16)
    real = lab != -1
    assert np.all(np.isinf(got["loss"][real])) and np.all(got["loss"][~real] == 0)
    n = np.linalg.norm(ref["dW"])
    assert n > 0 and np.linalg.norm(got["dW"] - ref["dW"]) <= (1e-2 if bf16 else 1e-5) * n


@pytest.mark.parametrize("bf16", [True, False])
def test_cross_entropy_of_large_scores(bf16):
    i = _ce_inputs(90, 64, 700, bf16, 5, spread=2000.0)       # differences of thousands: softmax is a choice
    ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], i["weight"])
    got = _run_ce(i, bf16)
    # scores of 10^4 in fp32: sums of 64 products, each off by 2^-24 of its size
    assert np.all(np.abs(got["loss"] - ref["loss"]) <= 2 * 80 * U24 * (np.abs(i["x"]) @ np.abs(i["W"])).max(1) + 1e-5)
    assert np.all(np.isfinite(got["dx"])) and np.all(np.isfinite(got["dW"]))
    n = np.linalg.norm(ref["dW"])
    assert np.linalg.norm(got["dW"] - ref["dW"]) <= 1e-2 * n


def test_cross_entropy_weights_of_any_sign_and_none():
    for bf16 in (True, False):
        i = _ce_inputs(120, 64, 130, bf16, 20)
        i["weight"][::4] = 0.0
        i["weight"][1::4] *= -1.0
        ref = O.cross_entropy(i["x"], i["W"], i["b"], i["labels"], i["weight"])
        _check_ce(_run_ce(i, bf16), i, ref, bf16)
        one = dict(i, weight=np.ones(120, dtype=np.float32))
        a, b = _run_ce(one, bf16), _run_ce(i, bf16, weight=False)
        for k in ("loss", "dx", "dW", "db"):
            np.testing.assert_array_equal(a[k], b[k])
        none = dict(i, b=None)
        ref = O.cross_entropy(i["x"], i["W"], None, i["labels"], i["weight"])
        got = _run_ce(none, bf16, want_db=False)
        assert got["db"] is None
        _check_ce(got, none, ref, bf16)


def test_cross_entropy_accumulates_parameter_gradients():
    torch = _torch()
    for bf16 in (True, False):
        for budget in (0, 1):
            i = _ce_inputs(600, 66, 130, bf16, 100)
            base = _run_ce(i, bf16, budget=budget)
            dt = torch.bfloat16 if bf16 else torch.float32
            dW, db = torch.full((66, 130), 3.0, device="cuda:0"), torch.full((130,), -2.0, device="cuda:0")
            Bd.run_ce_fwd_bwd(_dev(i["x"], dt), _dev(i["W"], dt), _dev(i["b"], torch.float32), _dev(i["labels"], torch.int32),
                              _dev(i["weight"], torch.float32), accumulate_into=(dW, db), budget_bytes=budget)
            # (fp32 additions in another order: a few half steps of the largest sum)
            np.testing.assert_allclose(_np(dW), base["dW"] + 3.0, atol=2e-6 * (3 + np.abs(base["dW"]).max()), rtol=0)
            np.testing.assert_allclose(_np(db), base["db"] - 2.0, atol=2e-6 * (2 + np.abs(base["db"]).max()), rtol=0)


# ---- as they are used ----------------------------------------------------------------------------------------------------------------------

def test_equal_calls_give_equal_bits():
    for bf16 in (True, False):
        i = _linear_inputs(900, 200, 300, bf16, res=True)
        a, b = (_run_linear(i, "gelu", 0.2, bf16) for _ in range(2))
        for k in a:
            np.testing.assert_array_equal(a[k], b[k])
        i = _ce_inputs(900, 200, 2000, bf16, 300)
        a, b = (_run_ce(i, bf16) for _ in range(2))
        for k in a:
            np.testing.assert_array_equal(a[k], b[k])


def _chain(dtype, seed=1):
    """A label encoder's step: widening layer, narrowing layer with the skip connection, cross entropy over the vocabulary."""
    torch = _torch()
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    n = lambda *s, k=1.0: (torch.randn(*s, generator=g, device="cuda:0") * k).to(dtype)
    B, U, D, F, V = 6, 35, 64, 200, 330
    p = dict(x=n(B, U, D), W1=n(D, F, k=D ** -0.5), b1=n(F, k=0.1), W2=n(F, D, k=F ** -0.5), b2=n(D, k=0.1), W_out=n(D, V, k=D ** -0.5), b_out=n(V, k=0.1))
    lab = torch.randint(0, V, (B, U), generator=g, device="cuda:0", dtype=torch.int32)
    for b in range(B):
        lab[b, U - 3 * b:] = -1
    w = torch.where(lab >= 0, 1.0 / float((lab >= 0).sum()), 0.0).float()
    rng = torch.tensor([5, 100], dtype=torch.int64, device="cuda:0")
    return p, lab, w, rng


def _chain_own(p, lab, w, rng, drop, reduction="sum"):
    from paper_2211_16270_amd import autograd as A
    h = A.rnnt_linear(p["x"], p["W1"], p["b1"], activation="silu", dropout=drop, rng_state=rng)
    rng[1] += 1                                               # (advanced between the layers, before the backward pass)
    y = A.rnnt_linear(h, p["W2"], p["b2"], residual=p["x"], dropout=drop, rng_state=rng)
    if reduction == "sum":
        return A.rnnt_ce_loss(y, p["W_out"], p["b_out"], lab, row_weight=w)
    return A.rnnt_ce_loss(y, p["W_out"], p["b_out"], lab, reduction="none")


def _chain_ref(p, lab, w, drop):
    torch = _torch()
    q = {k: v.detach().double().cpu().requires_grad_() for k, v in p.items()}
    B, U, D = q["x"].shape
    masks = [torch.from_numpy(O.keep_scale(B * U, n, 5, off, drop)).reshape(B, U, n) for n, off in ((q["W1"].shape[1], 100), (D, 101))]
    h = torch.nn.functional.silu(q["x"] @ q["W1"] + q["b1"]) * masks[0]
    y = (h @ q["W2"] + q["b2"]) * masks[1] + q["x"]
    logp = torch.log_softmax(y @ q["W_out"] + q["b_out"], dim=-1)
    at = lab.cpu().long().clamp(min=0)
    loss = (-logp.gather(-1, at.unsqueeze(-1)).squeeze(-1) * w.double().cpu()).sum()
    loss.backward()
    return float(loss), {k: v.grad.numpy() for k, v in q.items()}


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("reduction", ["sum", "none"])
def test_a_label_encoders_step_through_autograd(bf16, reduction):
    torch = _torch()
    p, lab, w, rng = _chain(torch.bfloat16 if bf16 else torch.float32)
    for v in p.values():
        v.requires_grad_()
    loss = _chain_own(p, lab, w, rng, 0.1, reduction)
    if reduction == "none":
        assert bool((loss[lab < 0] == 0).all())
        loss = (loss * w).sum()
    factor = 3.0
    (loss * factor).backward(retain_graph=True)
    ref, grads = _chain_ref(p, lab, w, 0.1)
    # (bf16: h and y are rounded between the layers; rms 2^-8 / sqrt(3) of scores of size one, averaged over rows)
    assert abs(float(loss) - ref) <= (5e-3 if bf16 else 1e-5) * abs(ref)
    first = {k: v.grad.clone() for k, v in p.items()}
    for k, v in p.items():
        assert v.grad.dtype == v.dtype
        e = np.linalg.norm(_np(v.grad) / factor - grads[k]) / np.linalg.norm(grads[k])
        # three layers' roundings of 2^-8 on the way (each 2.3e-3 rms at most, times the gain of the layer above)
        assert e <= (3e-2 if bf16 else 2e-5), (k, e)
    for v in p.values():
        v.grad = None
    (loss * factor).backward()                                # the graph once more: the cross entropy's gradients are computed again
    for k, v in p.items():
        e = np.linalg.norm(_np(v.grad) - _np(first[k])) / np.linalg.norm(_np(first[k]))
        assert e <= (1e-2 if bf16 else 1e-6), (k, e)


def test_layer_gradients_against_differences():
    torch = _torch()
    from paper_2211_16270_amd import autograd as A
    g = torch.Generator(device="cuda:0").manual_seed(4)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda:0")
    x, W, b, dy = n(20, 24), n(24, 16) * 0.2, n(16), n(20, 16)
    Wo, lab = n(16, 50) * 0.3, torch.randint(0, 50, (20,), generator=g, device="cuda:0", dtype=torch.int32)
    leaves = [x, W, b, Wo]
    for t in leaves:
        t.requires_grad_()

    def f():
        y = A.rnnt_linear(x, W, b, activation="tanh")
        return A.rnnt_ce_loss(y, Wo, None, lab)

    f().backward()
    for t in leaves:
        d = torch.randn(t.shape, generator=g, device="cuda:0")
        with torch.no_grad():
            t += 1e-2 * d
            up = float(f())
            t -= 2e-2 * d
            down = float(f())
            t += 1e-2 * d
        want = float((t.grad * d).sum())
        # second-order error of the difference and fp32 losses of size 80: 2^-24 * 80 * 4 / 2e-2
        assert abs((up - down) / 2e-2 - want) <= 2e-2 * abs(want) + 5e-2


def test_a_captured_step_replays_with_new_inputs_and_masks():
    torch = _torch()
    M, K, N, V = 150, 64, 96, 200
    g = torch.Generator(device="cuda:0").manual_seed(9)
    n = lambda *s, k=1.0: (torch.randn(*s, generator=g, device="cuda:0") * k).bfloat16()
    x, W, Wo = n(M, K), n(K, N, k=K ** -0.5), n(N, V, k=N ** -0.5)
    lab = torch.randint(-1, V, (M,), generator=g, device="cuda:0", dtype=torch.int32)
    rng = torch.tensor([1, 2], dtype=torch.int64, device="cuda:0")

    def step():
        f = Bd.run_linear_fwd(x, W, None, "gelu", dropout=0.3, rng_state=rng, save=True)
        o = Bd.run_ce_fwd_bwd(f["y"], Wo, None, lab)
        b = Bd.run_linear_bwd(x, W, o["dx"], "gelu", f["saved"], 0.3, f["rng_used"])
        rng.add_(1)
        return f["y"], o["loss"], o["dW"], b["dx"], b["dW"], b["db"]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for k in range(4):
        x.copy_(n(M, K))
        lab.copy_(torch.randint(-1, V, (M,), generator=g, device="cuda:0", dtype=torch.int32))
        rng.copy_(torch.tensor([50 + k, 60]))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert rng.tolist() == [51 + k, 61]          # (the step adds one to both)
        rng.copy_(torch.tensor([50 + k, 60]))
        want = step()
        for a, b in zip(got, want):
            assert torch.equal(a, b), k
        torch.zeros(1 << 20, device="cuda:0").sum().item()


def test_two_streams_at_once():
    torch = _torch()
    i = [_ce_inputs(700, 128, 1000, True, 100, seed=s) for s in range(2)]
    alone = [_run_ce(k, True) for k in i]
    streams = [torch.cuda.Stream() for _ in range(2)]
    dev = [(_dev(k["x"], torch.bfloat16), _dev(k["W"], torch.bfloat16), _dev(k["b"], torch.float32), _dev(k["labels"], torch.int32),
            _dev(k["weight"], torch.float32)) for k in i]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(3):
        for s in range(2):
            outs[s].append(Bd.run_ce_fwd_bwd(*dev[s], stream=streams[s]))
    torch.cuda.synchronize()
    for s in range(2):
        for o in outs[s]:
            for k in ("loss", "dx", "dW", "db"):
                np.testing.assert_array_equal(_np(o[k]), alone[s][k])


def test_views_and_leading_dimensions():
    torch = _torch()
    i = _linear_inputs(60, 63, 65, True, res=True)
    x, W, r = _dev(i["x"], torch.bfloat16), _dev(i["W"], torch.bfloat16), _dev(i["residual"], torch.bfloat16)
    want = Bd.run_linear_fwd(x, W, None, "silu", r)["y"]
    got = Bd.run_linear_fwd(x.view(3, 4, 5, 63), W, None, "silu", r.view(3, 4, 5, 65))["y"]
    assert got.shape == (3, 4, 5, 65) and torch.equal(got.view(60, 65), want)
    # a view that does not start on a 16-byte boundary
    big = torch.zeros(61 * 63, dtype=torch.bfloat16, device="cuda:0")
    big[63:] = x.reshape(-1)
    assert big[63:].data_ptr() % 16 != 0
    assert torch.equal(Bd.run_linear_fwd(big[63:].view(60, 63), W, None, "silu", r)["y"], want)
    with pytest.raises(ValueError, match="contiguous"):
        Bd.run_linear_fwd(x, W.t().contiguous().t(), None, "silu")
    with pytest.raises(ValueError, match="fit"):
        Bd.run_linear_fwd(x[:, :60].contiguous(), W)
    with pytest.raises(ValueError, match="dropout"):
        Bd.run_linear_fwd(x, W, dropout=0.1)
    with pytest.raises(ValueError, match="activation"):
        Bd.run_linear_fwd(x, W, activation="swish")
    with pytest.raises(ValueError, match="labels"):
        Bd.run_ce_fwd(x, W, None, torch.zeros(60, dtype=torch.int64, device="cuda:0"))
    with pytest.raises(ValueError, match="saved"):
        Bd.run_linear_bwd(x, W, want, "silu")


def test_scaling_and_totals():
    torch = _torch()
    i = _ce_inputs(333, 30, 77, True, 40)
    o = Bd.run_ce_fwd_bwd(_dev(i["x"], torch.bfloat16), _dev(i["W"], torch.bfloat16), None, _dev(i["labels"], torch.int32), param_grads_bf16=1)
    loss, w = o["loss"].clone(), _dev(i["weight"], torch.float32)
    loss[3], w[3] = float("inf"), 0.0
    want = float((loss.double() * w.double())[[k for k in range(333) if k != 3]].sum())
    assert abs(float(Bd.run_ce_total(loss, w)) - want) <= U24 * 2 * abs(want)
    before = {k: o[k].clone() for k in ("dx", "dW", "db")}
    Bd.run_ce_scale(torch.tensor(1.0, device="cuda:0"), o["dx"], o["dW"], o["db"])
    for k, v in before.items():
        assert torch.equal(o[k], v)
    Bd.run_ce_scale(torch.tensor(-2.5, device="cuda:0"), o["dx"], o["dW"], o["db"])
    for k, v in before.items():
        assert torch.equal(o[k], (v.float() * -2.5).to(v.dtype)), k
