"""Workspaces of the cross entropy for a budget: what the library names is what it takes, and a budget with room for a plan gets one that fits.  No GPU."""
import ctypes
import random

import pytest
import torch

from paper_2211_16270_amd import binding as Bd

# (R, D, V, bits, budget): sizes at which a plan's bytes fall as its chunks grow
NAMED = [(1024, 1024, 32768, 3, 97 << 20), (1024, 1024, 32768, 1, 102142720), (1856, 512, 1024, 3, 18881224), (1291, 685, 1343, 0, 27 << 20),
         (1742, 646, 717, 3, 12 << 20), (1130, 559, 898, 0, 15100000)]


def _desc(R, D, V, bits=0, dtype=Bd.RNNT_BF16):
    return Bd.RnntCeDesc(R, D, V, dtype, -1, 0, bits, 0)


def _bytes(d, budget, grads=True):
    return Bd.rnnt_ce_loss_workspace_bytes(d, grads, budget)


def _cases(n=4000):
    g = random.Random(11)
    for R, D, V, bits, budget in NAMED:
        yield _desc(R, D, V, bits), True, budget
    for _ in range(n):
        dtype = g.choice((Bd.RNNT_BF16, Bd.RNNT_BF16, Bd.RNNT_F32))
        size = lambda lo, hi: int(lo * (hi / lo) ** g.random())
        d = _desc(size(1, 60000), size(1, 1200), size(1, 40000), g.randrange(4) if dtype == Bd.RNNT_BF16 else 0, dtype)
        yield d, g.random() < 0.7, size(1 << 16, 4 << 30)


def test_a_size_that_the_library_names_is_a_budget_for_itself():
    for d, grads, budget in _cases():
        n = _bytes(d, budget, grads)
        assert n > 0 and _bytes(d, n, grads) == n, (d.R, d.D, d.V, d.dtype, d.param_grads_bf16, grads, budget)


def test_a_budget_with_room_for_a_plan_is_kept():
    for d, grads, budget in _cases():
        what = (d.R, d.D, d.V, d.dtype, d.param_grads_bf16, grads, budget)
        n, default, least = _bytes(d, budget, grads), _bytes(d, 0, grads), _bytes(d, 1, grads)
        assert least <= min(n, default), what
        if budget >= least:
            assert n <= budget, what
        else:
            assert n == least, what
        assert _bytes(d, default, grads) <= default, what
        # what fits a budget fits a larger one too
        assert _bytes(d, budget + budget // 3, grads) <= max(least, budget + budget // 3), what


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls' pointers are none: only without a GPU do they end at the first launch")
def test_a_call_takes_every_size_that_the_library_names():
    L, P = Bd.lib(), ctypes.c_void_p(0x1000)
    refused = Bd.STATUS_NAMES.index("RNNT_ERR_WORKSPACE")
    for k, (d, grads, budget) in enumerate(_cases(400)):
        n = _bytes(d, budget, grads)
        for more in (0, 256, n // 2):
            if grads:
                st = L.rnnt_ce_loss_fwd_bwd(ctypes.byref(d), P, P, P, P, P, P, P, P, P, P, n + more, None)
            else:
                st = L.rnnt_ce_loss_fwd(ctypes.byref(d), P, P, P, P, P, P, n + more, None)
            assert st != refused, (d.R, d.D, d.V, d.dtype, d.param_grads_bf16, grads, budget, more)
