"""Host side of the layers beside the transducer loss: exported symbols, descriptors, refusals, workspace sizes.  No GPU: every refusal here
happens before a launch."""
import ctypes
import os
import re

import numpy as np
import pytest

from paper_2211_16270_amd import binding as Bd
from tests import layer_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)


def test_library_exports_what_the_header_of_the_layers_declares():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rnnt_layers.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(rnnt_[a-z_0-9]+)\s*\(", text))
    assert declared == set(Bd.LAYER_EXPORTS)
    for name in declared:
        assert hasattr(Bd.lib(), name), name


def test_descriptor_layouts_match_the_header():
    assert ctypes.sizeof(Bd.RnntLinearDesc) == 40
    assert ctypes.sizeof(Bd.RnntCeDesc) == 40


def _linear(**kw):
    d = dict(M=100, K=64, N=64, dtype=1, activation=0, dropout=0.0, accumulate_params=0, param_grads_bf16=0, bias_bf16=0)
    d.update(kw)
    return Bd.RnntLinearDesc(*d.values())


def _ce(**kw):
    d = dict(R=100, D=64, V=64, dtype=1, ignore_label=-1, accumulate_params=0, param_grads_bf16=0, bias_bf16=0)
    d.update(kw)
    return Bd.RnntCeDesc(*d.values())


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), "SHAPE"), (dict(M=(1 << 30) + 1), "SHAPE"), (dict(K=0), "SHAPE"), (dict(N=0), "SHAPE"), (dict(K=(1 << 20) + 1), "SHAPE"),
    (dict(N=(1 << 20) + 1), "SHAPE"), (dict(dropout=1.0), "SHAPE"), (dict(dropout=-0.1), "SHAPE"), (dict(dropout=float("nan")), "SHAPE"),
    (dict(dtype=2), "UNSUPPORTED"), (dict(activation=5), "UNSUPPORTED"), (dict(activation=-1), "UNSUPPORTED"), (dict(bias_bf16=2), "SHAPE"),
])
def test_linear_descriptors_out_of_range_are_refused(kw, status):
    want = Bd.STATUS_NAMES.index("RNNT_ERR_" + status)
    d = _linear(**kw)
    L = Bd.lib()
    assert L.rnnt_linear_fwd(ctypes.byref(d), PTR, PTR, PTR, None, PTR, None, PTR, None, PTR, 1 << 40, None) == want
    assert L.rnnt_linear_bwd(ctypes.byref(d), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 40, None) == want
    assert Bd.rnnt_linear_workspace_bytes(d, False) == 0 and Bd.rnnt_linear_workspace_bytes(d, True) == 0


def test_linear_calls_are_refused_before_a_launch():
    L, S = Bd.lib(), {n[9:]: i for i, n in enumerate(Bd.STATUS_NAMES)}

    def fwd(d, x=PTR, W=PTR, b=PTR, res=None, rng=None, used=None, y=PTR, saved=None, ws=PTR, n=1 << 40):
        return L.rnnt_linear_fwd(ctypes.byref(d) if d is not None else None, x, W, b, res, rng, used, y, saved, ws, n, None)

    def bwd(d, x=PTR, W=PTR, saved=PTR, rng=None, dy=PTR, dx=PTR, dW=PTR, db=PTR, ws=PTR, n=1 << 40):
        return L.rnnt_linear_bwd(ctypes.byref(d), x, W, saved, rng, dy, dx, dW, db, ws, n, None)

    d = _linear()
    assert fwd(None) == S["NULL"] and fwd(d, x=None) == S["NULL"] and fwd(d, W=None) == S["NULL"] and fwd(d, y=None) == S["NULL"]
    assert fwd(_linear(dropout=0.5)) == S["NULL"] and fwd(d, used=PTR) == S["NULL"]
    for k in ("x", "W", "b", "res", "y", "saved"):
        assert fwd(d, **{k: ODD}) == S["UNSUPPORTED"], k
    assert fwd(_linear(dropout=0.5), rng=ODD) == S["UNSUPPORTED"]
    odd = _linear(M=100, K=63, N=65)
    need = Bd.rnnt_linear_workspace_bytes(odd, False)
    assert need > 0
    assert fwd(odd, n=need - 1) == S["WORKSPACE"] and fwd(odd, ws=None) == S["WORKSPACE"] and fwd(odd, ws=ctypes.c_void_p(0x1010)) == S["WORKSPACE"]
    assert bwd(d, x=None) == S["NULL"] and bwd(d, dy=None) == S["NULL"] and bwd(_linear(activation=1), saved=None) == S["NULL"]
    assert bwd(_linear(dropout=0.5)) == S["NULL"]
    assert bwd(d, ws=None) == S["WORKSPACE"]
    for k in ("x", "W", "saved", "dy", "dx", "dW", "db"):
        assert bwd(d, **{k: ODD}) == S["UNSUPPORTED"], k
    assert bwd(_linear(dtype=0, param_grads_bf16=1)) == S["UNSUPPORTED"]
    assert bwd(_linear(param_grads_bf16=1, accumulate_params=1)) == S["UNSUPPORTED"]
    assert bwd(_linear(param_grads_bf16=4)) == S["SHAPE"] and bwd(_linear(accumulate_params=2)) == S["SHAPE"]


@pytest.mark.parametrize("kw,status", [
    (dict(R=-1), "SHAPE"), (dict(R=(1 << 30) + 1), "SHAPE"), (dict(D=0), "SHAPE"), (dict(V=0), "SHAPE"), (dict(V=(1 << 20) + 1), "SHAPE"),
    (dict(dtype=7), "UNSUPPORTED"), (dict(bias_bf16=-1), "SHAPE"),
])
def test_cross_entropy_descriptors_out_of_range_are_refused(kw, status):
    want = Bd.STATUS_NAMES.index("RNNT_ERR_" + status)
    d = _ce(**kw)
    L = Bd.lib()
    assert L.rnnt_ce_loss_fwd(ctypes.byref(d), PTR, PTR, PTR, PTR, PTR, PTR, 1 << 40, None) == want
    assert L.rnnt_ce_loss_fwd_bwd(ctypes.byref(d), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 40, None) == want
    assert Bd.rnnt_ce_loss_workspace_bytes(d, False) == 0 and Bd.rnnt_ce_loss_workspace_bytes(d, True) == 0


def test_cross_entropy_calls_are_refused_before_a_launch():
    L, S = Bd.lib(), {n[9:]: i for i, n in enumerate(Bd.STATUS_NAMES)}

    def call(d, x=PTR, W=PTR, b=PTR, label=PTR, weight=PTR, loss=PTR, dx=PTR, dW=PTR, db=PTR, ws=PTR, n=1 << 40):
        return L.rnnt_ce_loss_fwd_bwd(ctypes.byref(d), x, W, b, label, weight, loss, dx, dW, db, ws, n, None)

    d = _ce()
    for k in ("x", "W", "label", "loss", "dx", "dW"):
        assert call(d, **{k: None}) == S["NULL"], k
    for k in ("x", "W", "b", "dx", "dW", "db"):
        assert call(d, **{k: ODD}) == S["UNSUPPORTED"], k
    for k in ("label", "weight", "loss"):
        assert call(d, **{k: ctypes.c_void_p(0x1002)}) == S["UNSUPPORTED"], k
    smallest = Bd.rnnt_ce_loss_workspace_bytes(d, True, 1)
    assert call(d, n=smallest - 1) == S["WORKSPACE"] and call(d, ws=None) == S["WORKSPACE"] and call(d, n=0) == S["WORKSPACE"]
    assert call(_ce(dtype=0, param_grads_bf16=1)) == S["UNSUPPORTED"]
    assert call(_ce(param_grads_bf16=2, accumulate_params=1)) == S["UNSUPPORTED"]
    assert L.rnnt_ce_loss_total(ctypes.byref(d), None, None, PTR, None) == S["NULL"]
    assert L.rnnt_ce_loss_total(ctypes.byref(d), PTR, None, None, None) == S["NULL"]
    assert L.rnnt_ce_loss_scale(ctypes.byref(d), None, PTR, PTR, PTR, None) == S["NULL"]
    assert L.rnnt_ce_loss_scale(ctypes.byref(d), PTR, ODD, PTR, PTR, None) == S["UNSUPPORTED"]


def test_cross_entropy_workspaces_follow_their_budget():
    for dtype in (0, 1):
        d = _ce(R=50000, D=512, V=32768, dtype=dtype)
        smallest, default = Bd.rnnt_ce_loss_workspace_bytes(d, True, 1), Bd.rnnt_ce_loss_workspace_bytes(d, True)
        assert 0 < smallest < default < 3 << 30
        for budget in (smallest, smallest + (64 << 20), default, 2 * default, 8 * default):
            assert Bd.rnnt_ce_loss_workspace_bytes(d, True, budget) <= budget
        # the scores as a whole would take 50000 x 32768
        assert Bd.rnnt_ce_loss_workspace_bytes(d, True, 1) < 50000 * 32768
        assert Bd.rnnt_ce_loss_workspace_bytes(d, False) < default


def test_partial_sums_of_any_fewer_rows_fit(tmp_path):
    import shutil
    import subprocess
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    src = tmp_path / "t.cpp"
    src.write_text('#include "%s"\n' % os.path.join(ROOT, "paper_2211_16270_amd", "csrc", "layers.h") + r"""
#include <cstdio>
#include <random>
int main() {
    std::mt19937_64 g(5);
    for (int i = 0; i < 400000; ++i) {
        const long long most = i % 3 == 0 ? 300 : i % 3 == 1 ? 40000 : 3000000, rows = g() % (most + 1), fewer = g() % (rows + 1);
        const long long cols = 1 + g() % (i % 2 ? 3000 : 70000);
        if (rnnt::sum_blocks(fewer, cols) > rnnt::sum_capacity(rows, cols)) { std::printf("%lld %lld %lld\n", rows, fewer, cols); return 1; }
        if (rnnt::sum_rows(rows, cols) % 16 != 0 || rnnt::sum_rows(rows, cols) > 128) return 2;
    }
    return 0;
}
""")
    exe = tmp_path / "t"
    subprocess.run([gxx, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-w", "-o", str(exe), str(src)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_philox_of_the_oracle_against_published_numbers():
    # Random123's known answers of Philox4x32-10: counter and key all zeros, all ones
    bits = O.philox16(1, 8, 0, 0)[0]
    words = [int(bits[2 * j] | bits[2 * j + 1] << 16) for j in range(4)]
    assert words == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]


def test_oracle_gradients_against_differences():
    g = np.random.default_rng(3)
    for name in Bd.ACTIVATIONS:
        x, W, b, dy = g.normal(size=(4, 5)), g.normal(size=(5, 3)), g.normal(size=3), g.normal(size=(4, 3))
        keep = O.keep_scale(4, 3, 11, 12, 0.3)
        out = O.linear(x, W, b, name, None, keep, dy)
        for arr, grad in ((x, out["dx"]), (W, out["dW"]), (b, out["db"])):
            i = tuple(int(g.integers(n)) for n in arr.shape)
            f = []
            for s in (1e-6, -1e-6):
                arr[i] += s
                f.append((O.linear(x, W, b, name, None, keep)["y"] * dy).sum())
                arr[i] -= s
            assert abs((f[0] - f[1]) / 2e-6 - grad[i]) < 1e-6 * max(1.0, abs(grad[i])), name
    x, W, b, w = g.normal(size=(6, 4)), g.normal(size=(4, 7)), g.normal(size=7), g.normal(size=6)
    lab = np.array([0, 6, -1, 3, 2, -1])
    out = O.cross_entropy(x, W, b, lab, w)
    assert out["loss"][2] == 0 and np.all(out["dx"][2] == 0)
    for arr, grad in ((x, out["dx"]), (W, out["dW"]), (b, out["db"])):
        i = tuple(int(g.integers(n)) for n in arr.shape)
        f = []
        for s in (1e-6, -1e-6):
            arr[i] += s
            f.append((O.cross_entropy(x, W, b, lab, w)["loss"] * w).sum())
            arr[i] -= s
        assert abs((f[0] - f[1]) / 2e-6 - grad[i]) < 1e-6 * max(1.0, abs(grad[i]))


def test_python_front_end_refuses_tensors_that_do_not_fit():
    import torch
    from paper_2211_16270_amd import autograd as A
    x, W = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.run_linear_fwd(x, W)
    with pytest.raises(ValueError, match="CUDA"):
        Bd.run_ce_fwd(x, W, None, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="reduction"):
        A.rnnt_ce_loss(x, W, None, torch.zeros(4, dtype=torch.int32), reduction="mean")
    with pytest.raises(ValueError, match="row_weight"):
        A.rnnt_ce_loss(x, W, None, torch.zeros(4, dtype=torch.int32), row_weight=torch.ones(4), reduction="none")
