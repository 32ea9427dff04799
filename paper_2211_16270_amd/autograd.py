"""torch.autograd front end of the C-ABI library (argument marshalling only: every number comes out of
the library's calls).

    loss = rnnt_joint_loss(enc, pred, W_out, b_out, labels, T_len, U_len, blank=0)     # [B], -ln P(y_b|x_b)
    loss.sum().backward()        # or loss.mean(), (loss * mask).sum(), ...

The library computes the loss and all gradients in one call (Algorithm 1 of the paper: the gradients of the
output layer are accumulated while the samples are walked, nothing is kept for a later backward pass), so the
forward of the autograd function already holds the gradients of sum_b w_b loss_b for the weights w it was
given (default: ones).  backward() hands them out if the incoming gradient of the loss vector equals those
weights, and otherwise calls the library once more with the incoming gradient as the weights.  Pass
`sample_weight` (e.g. 1/B for a mean) to make the first call the only one.  The weights of the library are
non-negative, so the gradient that reaches the loss vector must be >= 0 for every sample (backward raises
otherwise).  The forward call's outputs and workspace stay alive until backward has run.

    y = rnnt_linear(x, W, b, activation="silu", residual=None, dropout=0.1, rng_state=state)      # the encoders' layers
    loss = rnnt_ce_loss(x, W_out, b_out, labels, row_weight=w)                                    # cross entropy of the same output layer

Steps of these can be captured into a graph (torch.cuda.graph), forward and backward passes together or each in one of its own.  Torch's own condition holds: no
eager graph of the same leaves may be alive then (delete the warm-up's outputs and losses before the capture), as its gradient accumulators belong to another
stream.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as Bd


class _RnntJointLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, enc, pred, W_out, b_out, labels, T_len, U_len, blank, sample_weight, workspace, keep_scores):
        if not (enc.is_cuda and enc.is_contiguous() and pred.is_contiguous() and W_out.is_contiguous()):
            raise ValueError("enc, pred, W_out must be contiguous CUDA tensors")
        B, T_max, H = enc.shape
        U_max = pred.shape[1] - 1
        V = W_out.shape[1]
        dtype = Bd.RNNT_BF16 if enc.dtype == torch.bfloat16 else Bd.RNNT_F32
        T_host = np.ascontiguousarray(T_len, dtype=np.int32)
        U_host = np.ascontiguousarray(U_len, dtype=np.int32)
        w_host = np.ones(B, dtype=np.float32) if sample_weight is None else \
            np.ascontiguousarray(sample_weight, dtype=np.float32)
        dev = dict(enc=enc, pred=pred, W_out=W_out, b_out=b_out, labels=labels, T_len=T_host, U_len=U_host)
        shape = (B, T_max, U_max, H, V, int(blank), dtype)
        # bf16 leaves get bf16 gradients: the library rounds them itself instead of a conversion pass here
        opts = dict(keep_scores=int(keep_scores), input_grads_bf16=int(dtype == Bd.RNNT_BF16))
        out = Bd.run_fwd_bwd(dev, *shape, workspace=workspace, sample_weight=w_host, **opts)
        ctx.dev, ctx.shape, ctx.w_host, ctx.out, ctx.opts = dev, shape, w_host, out, opts
        ctx.mark_non_differentiable(labels)
        return out["loss"]

    @staticmethod
    def backward(ctx, grad_loss):
        g = grad_loss.detach().float().cpu().numpy()          # B numbers; also orders this after the forward
        if not (np.all(np.isfinite(g)) and np.all(g >= 0.0)):
            # the library takes one weight >= 0 per sample (they scale posterior probabilities in log space)
            raise ValueError("rnnt_joint_loss: the gradient reaching the loss vector must be finite and >= 0 for "
                             "every sample (sum, mean, masks and positive scalings are; a negated loss is not)")
        out = ctx.out
        if not np.array_equal(g, ctx.w_host):
            out = Bd.run_fwd_bwd(ctx.dev, *ctx.shape, workspace=ctx.out["workspace"], sample_weight=g, **ctx.opts)
        enc, W_out, b_out = ctx.dev["enc"], ctx.dev["W_out"], ctx.dev["b_out"]
        return (out["d_enc"].to(enc.dtype), out["d_pred"].to(enc.dtype), out["dW_out"].to(W_out.dtype),
                out["db_out"].to(b_out.dtype), None, None, None, None, None, None, None)


def rnnt_joint_loss(enc, pred, W_out, b_out, labels, T_len, U_len, blank: int = 0, sample_weight=None,
                    workspace=None, keep_scores: bool = False):
    """Per-sample transducer loss [B] with gradients for enc, pred, W_out, b_out.

    enc [B,T_max,H], pred [B,U_max+1,H], W_out [H,V] (float32 or bfloat16, CUDA, contiguous), b_out [V] float32,
    labels [B,U_max] int32 on the device, T_len / U_len host arrays of B int32.  sample_weight: host array of B
    non-negative floats, the weights the loss vector is going to be summed with (None: ones).  keep_scores
    (bfloat16 only): the descriptor field of that name, scores kept in a larger workspace instead of computed twice."""
    return _RnntJointLoss.apply(enc, pred, W_out, b_out, labels, T_len, U_len, blank, sample_weight, workspace,
                                keep_scores)


def _tracked(*tensors):
    """Whether a gradient of one of them can be asked for.  (ctx.needs_input_grad does not tell: it is true under no_grad too.)"""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _grads_bf16(W, b):
    """param_grads_bf16 of leaves W, b: gradients of their types"""
    return 0 if W.dtype == torch.float32 else 3 if b is not None and b.dtype == torch.bfloat16 else 1


class _RnntLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, b, activation, residual, dropout, rng_state):
        # (with dropout the call also leaves the state its kernels saw: the caller may advance it before the backward pass)
        out = Bd.run_linear_fwd(x, W, b, activation, residual, dropout, rng_state, save=any(ctx.needs_input_grad[:3]))
        ctx.save_for_backward(x, W, out["saved"], out["rng_used"])
        ctx.opts = activation, dropout, None if b is None else b.dtype, _grads_bf16(W, b)
        return out["y"]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, W, saved, rng = ctx.saved_tensors
        activation, dropout, b_dtype, bits = ctx.opts
        need = ctx.needs_input_grad
        want = tuple(k for k, n in zip(("dx", "dW", "db"), need) if n)
        dx = dW = db = None
        dy = dy.contiguous()
        if want:
            g = Bd.run_linear_bwd(x, W, dy, activation, saved, dropout, rng, param_grads_bf16=bits, want=want)
            dx, dW, db = g["dx"], g["dW"], g["db"]
            if db is not None and db.dtype != b_dtype:
                db = db.to(b_dtype)
        return dx, dW, db, None, dy if need[4] else None, None, None


def rnnt_linear(x, W, b=None, activation="none", residual=None, dropout: float = 0.0, rng_state=None):
    """residual + dropout(act(x W + b)) with gradients for x, W, b and residual.

    x [..., K], W [K, N] (float32 or bfloat16, CUDA, contiguous), b [N] (float32 or bfloat16) or None, residual [..., N] or None; activation: none,
    relu, silu, gelu, tanh.  dropout in [0, 1) needs rng_state, an int64 tensor [2] on the device with {seed, offset}: the mask is a function of them
    and of an entry's place, so advance the offset between calls that shall have different masks (in place, also inside a captured graph)."""
    if not _tracked(x, W, b, residual):
        return Bd.run_linear_fwd(x, W, b, activation, residual, dropout, rng_state)["y"]
    return _RnntLinear.apply(x, W, b, activation, residual, float(dropout), rng_state)


def _ce_grads(x, W, b, labels, row_weight, ignore_label, budget_bytes):
    return Bd.run_ce_fwd_bwd(x, W, b, labels, row_weight, ignore_label, param_grads_bf16=_grads_bf16(W, b), want_db=b is not None,
                             budget_bytes=budget_bytes)


def _ce_leaf_grads(need, out, b):
    """dx, dW, db as the leaves have them (the library's db is float32 beside a float32 W, whatever b's type)"""
    db = out["db"]
    if need[2] and db.dtype != b.dtype:
        db = db.to(b.dtype)
    return out["dx"] if need[0] else None, out["dW"] if need[1] else None, db if need[2] else None


class _RnntCeSum(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, b, labels, row_weight, ignore_label, budget_bytes):
        out = _ce_grads(x, W, b, labels, row_weight, ignore_label, budget_bytes)
        ctx.save_for_backward(x, W, b, labels, row_weight)
        ctx.grads, ctx.opts, ctx.captured = out, (ignore_label, budget_bytes), Bd.capture_id()
        return Bd.run_ce_total(out["loss"], row_weight)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        x, W, b, labels, row_weight = ctx.saved_tensors
        g = g.float().contiguous()
        capture = Bd.capture_id()
        if ctx.grads is not None and ctx.captured == capture:
            # the forward call's gradients are handed out, times g in place; a second backward pass of the same graph computes them again, and so does one
            # that is captured behind an eager forward call
            out, ctx.grads = ctx.grads, None
            Bd.run_ce_scale(g, out["dx"], out["dW"], out["db"])
        elif ctx.grads is not None and ctx.captured and capture:
            # captured, and the forward call too, but elsewhere: in place, each replay of this graph alone would scale them once more
            out = {k: None if ctx.grads[k] is None else ctx.grads[k].clone() for k in ("dx", "dW", "db")}
            Bd.run_ce_scale(g, out["dx"], out["dW"], out["db"])
        else:
            w = g.expand(labels.shape).contiguous() if row_weight is None else row_weight * g
            out = _ce_grads(x, W, b, labels, w, *ctx.opts)
        return (*_ce_leaf_grads(ctx.needs_input_grad, out, b), None, None, None, None)


class _RnntCeRows(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, b, labels, ignore_label, budget_bytes):
        ctx.save_for_backward(x, W, b, labels)
        ctx.opts = ignore_label, budget_bytes
        return Bd.run_ce_fwd(x, W, b, labels, ignore_label, budget_bytes=budget_bytes)["loss"]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        x, W, b, labels = ctx.saved_tensors
        out = _ce_grads(x, W, b, labels, g.float().contiguous(), *ctx.opts)
        return (*_ce_leaf_grads(ctx.needs_input_grad, out, b), None, None, None)


def rnnt_ce_loss(x, W, b, labels, row_weight=None, ignore_label: int = -1, reduction: str = "sum", budget_bytes: int = 0):
    """Cross entropy of softmax(x W + b) with gradients for x, W and b, without the [rows, V] scores.

    x [..., D], W [D, V] (float32 or bfloat16, CUDA, contiguous), b [V] (float32 or bfloat16) or None, labels [...] int32 (rows with ignore_label are
    padding: loss and gradients 0, x never used).
    reduction "sum": sum of row_weight * loss over the rows (row_weight [...] float32 on the device, without a gradient of its own, None: ones; 1 / count for
    a mean), a scalar.  The forward call computes the gradients too (three products per row) where one can be asked for, not under no_grad; backward scales them, which
    rounds those of bfloat16 leaves a second time unless the incoming gradient is a power of two (1 with loss.backward(); put other factors into row_weight).
    reduction "none": the loss of each row; the gradients are computed in backward, with the incoming gradient as the rows' weights (four products)."""
    if reduction not in ("sum", "none"):
        raise ValueError(f"reduction must be 'sum' or 'none', got {reduction!r}")
    if reduction == "none" and row_weight is not None:
        raise ValueError("row_weight goes with reduction='sum'; with 'none' weight the returned losses")
    if _tracked(row_weight):
        raise ValueError("row_weight gets no gradient here: pass it detached, or weight the losses of reduction='none'")
    if not _tracked(x, W, b):
        loss = Bd.run_ce_fwd(x, W, b, labels, ignore_label, budget_bytes=budget_bytes)["loss"]
        return loss if reduction == "none" else Bd.run_ce_total(loss, row_weight)
    if reduction == "sum":
        return _RnntCeSum.apply(x, W, b, labels, row_weight, ignore_label, budget_bytes)
    return _RnntCeRows.apply(x, W, b, labels, ignore_label, budget_bytes)
