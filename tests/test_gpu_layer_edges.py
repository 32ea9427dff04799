"""Calls at the edges of the layers beside the transducer loss, on the GPU: empty batches, streams, graphs, evaluation, mixed types."""
import numpy as np
import pytest

from paper_2211_16270_amd import binding as Bd
from tests import layer_oracle as O
from tests.test_gpu_layers import _ce_inputs, _check_ce, _check_linear, _dev, _linear_inputs, _np, _torch

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
