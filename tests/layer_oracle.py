"""The layers beside the transducer loss in 64 bits, written from their formulas (CPU, numpy)."""
import math

import numpy as np

_erf = np.vectorize(math.erf)


def philox16(M, N, seed, offset):
    """The 16 random bits of each entry (m, n): Philox4x32-10, key = seed, counter = (n / 8, m, offset), half n % 2 of word (n % 8) / 2."""
    mask = 0xFFFFFFFF
    c = np.zeros((M, (N + 7) // 8, 4), dtype=np.uint64)
    c[..., 0] = np.arange((N + 7) // 8, dtype=np.uint64)[None, :]
    c[..., 1] = np.arange(M, dtype=np.uint64)[:, None]
    c[..., 2], c[..., 3] = offset & mask, (offset >> 32) & mask
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        p0, p1 = c[..., 0] * np.uint64(0xD2511F53), c[..., 2] * np.uint64(0xCD9E8D57)
        c = np.stack([(p1 >> np.uint64(32)) ^ c[..., 1] ^ np.uint64(k0), p1 & np.uint64(mask),
                      (p0 >> np.uint64(32)) ^ c[..., 3] ^ np.uint64(k1), p0 & np.uint64(mask)], axis=-1)
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    halves = np.stack([c & np.uint64(0xFFFF), c >> np.uint64(16)], axis=-1)
    return halves.reshape(M, -1)[:, :N].astype(np.int64)


def keep_scale(M, N, seed, offset, p):
    cut = min(65535, round(p * 65536))
    if cut == 0:
        return np.ones((M, N))
    return np.where(philox16(M, N, seed, offset) >= cut, 65536.0 / (65536 - cut), 0.0)


def act(z, name):
    """act(z), act'(z)"""
    if name == "none":
        return z, np.ones_like(z)
    if name == "relu":
        return np.where(z < 0, 0.0, z), (z > 0).astype(z.dtype)
    if name == "tanh":
        t = np.tanh(z)
        return t, 1.0 / np.cosh(np.clip(z, -300, 300)) ** 2
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-np.clip(z, -700, 700)))
        return z * s, s * (1.0 + z * (1.0 - s))
    phi = 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
    return z * phi, phi + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)


def linear(x, W, b, name="none", residual=None, keep=None, dy=None):
    z = x @ W + (0.0 if b is None else b)
    a, da = act(z, name)
    if keep is not None:
        a = a * keep
    out = dict(z=z, y=a if residual is None else a + residual)
    if dy is not None:
        dz = dy * da
        if keep is not None:
            dz = dz * keep
        out.update(dz=dz, dx=dz @ W.T, dW=x.T @ dz, db=dz.sum(0))
    return out


def cross_entropy(x, W, b, labels, weight=None, ignore=-1):
    R, V = x.shape[0], W.shape[1]
    real = labels != ignore
    w = (np.ones(R) if weight is None else weight.astype(np.float64)) * real
    h = np.where(real[:, None], x, 0.0) @ W + (0.0 if b is None else b)
    top = h.max(1, keepdims=True)
    top = np.where(np.isinf(top), 0.0, top)
    e = np.exp(h - top)
    total = e.sum(1, keepdims=True)
    known = real & (labels >= 0) & (labels < V)
    at = np.where(known, labels, 0)
    with np.errstate(divide="ignore", invalid="ignore"):
        loss = np.where(real, np.where(known & (total[:, 0] > 0), top[:, 0] + np.log(total[:, 0]) - h[np.arange(R), at], np.inf), 0.0)
        p = np.where(total > 0, e / total, 0.0)
    dh = w[:, None] * p
    dh[np.arange(R)[known], at[known]] -= w[known]
    return dict(h=h, loss=loss, dh=dh, dx=dh @ W.T, dW=np.where(real[:, None], x, 0.0).T @ dh, db=dh.sum(0))
