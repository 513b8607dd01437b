"""Operators of a decoder layer's residual chain in plain numpy: linear attention with a decay for each head, dropout from a
counter-based generator, and the root-mean-square norm of a residual sum.  TEST INFRASTRUCTURE ONLY (see ops.py)."""
from __future__ import annotations

import numpy as np


# ----------------------------------------------------------------------------- linear attention
def _powers(log_decay, dtype):
    return np.exp(np.asarray(log_decay, dtype))            # exp(-inf) = 0


def linear_attention_fwd(q, k, v, log_decay, s0=None, lens=None):
    """q, k, v [B, H, S, dh]; the recurrence, one position after another.  Returns o and the last state [B, H, dh, dh]."""
    B, H, S, dh = q.shape
    lam = _powers(log_decay, q.dtype)[None, :, None, None]
    s = np.zeros((B, H, dh, dh), q.dtype) if s0 is None else s0.astype(q.dtype).copy()
    n = np.full(B, S) if lens is None else np.clip(lens, 0, S)
    o = np.zeros_like(q)
    for t in range(S):
        live = (t < n)
        s[live] = (lam * s + k[:, :, t, :, None] * v[:, :, t, None, :])[live]
        o[live, :, t] = (q[:, :, t, None, :] @ s)[live][..., 0, :] / np.sqrt(dh)
    return o, s


def linear_attention_bwd(q, k, v, log_decay, do, s0=None, ds_out=None, lens=None):
    """The recurrence's adjoint, from the last position to the first.  Returns dq, dk, dv, ds0."""
    B, H, S, dh = q.shape
    lam = _powers(log_decay, q.dtype)[None, :, None, None]
    n = np.full(B, S) if lens is None else np.clip(lens, 0, S)
    states, s = [], np.zeros((B, H, dh, dh), q.dtype) if s0 is None else s0.astype(q.dtype).copy()
    for t in range(S):
        live = (t < n)
        s = s.copy()
        s[live] = (lam * s + k[:, :, t, :, None] * v[:, :, t, None, :])[live]
        states.append(s)
    ds = np.zeros((B, H, dh, dh), q.dtype) if ds_out is None else ds_out.astype(q.dtype).copy()
    dq, dk, dv = np.zeros_like(q), np.zeros_like(q), np.zeros_like(q)
    for t in reversed(range(S)):
        live = (t < n)
        g = do[:, :, t] / np.sqrt(dh)
        full = ds + q[:, :, t, :, None] * g[:, :, None, :]
        dq[live, :, t] = (states[t] @ g[..., None])[live][..., 0]
        dk[live, :, t] = (full @ v[:, :, t, :, None])[live][..., 0]
        dv[live, :, t] = (k[:, :, t, None, :] @ full)[live][..., 0, :]
        ds[live] = (lam * full)[live]
    return dq, dk, dv, ds


# ----------------------------------------------------------------------------- dropout
def philox(counter, key):
    """Philox4x32-10 (Salmon, Moraes, Dror and Shaw, 2011); counter [..., 4] and key [2] of 32-bit numbers."""
    c = [np.asarray(counter[..., i], np.uint64) for i in range(4)]
    k = [np.uint64(key[0]), np.uint64(key[1])]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    with np.errstate(over="ignore"):
        for _ in range(10):
            a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(b >> half) ^ c[1] ^ k[0], b & low, (a >> half) ^ c[3] ^ k[1], a & low]
            k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return np.stack(c, -1).astype(np.uint32)


def dropout_threshold(p):
    """Of 65536: numbers below it are dropped.  p as the 32-bit number that the call receives."""
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def dropout_kept(n, p, seed, step, site):
    """Which of n elements are kept: element 8 i + j has the j-th 16-bit half of counter (i, site, step)."""
    groups = -(-n // 8)
    c = np.zeros((groups, 4), np.uint64)
    c[:, 0], c[:, 1], c[:, 2], c[:, 3] = np.arange(groups), site, step & 0xFFFFFFFF, step >> 32
    w = philox(c, (seed & 0xFFFFFFFF, seed >> 32))
    u = np.stack([w & 0xFFFF, w >> 16], -1).reshape(-1)[:n]
    return u >= dropout_threshold(p)


def dropout(x, p, seed, step, site):
    """Its own gradient: the same call on dy."""
    thr = dropout_threshold(p)
    if thr == 0:
        return x.copy()
    kept = dropout_kept(x.size, p, seed, step, site).reshape(x.shape)
    return np.where(kept, x * (65536.0 / (65536.0 - thr) if thr < 65536 else 0.0), 0.0)


# ----------------------------------------------------------------------------- RMS norm
def rmsnorm_fwd(r, g, eps):
    """Returns y and the rows' reciprocal root mean squares."""
    rstd = 1.0 / np.sqrt((r * r).mean(-1) + eps)
    return r * rstd[:, None] * g, rstd


def rmsnorm_bwd(dy, r, rstd, g):
    """Returns dr and dg."""
    xhat, a = r * rstd[:, None], dy * g
    return rstd[:, None] * (a - xhat * (a * xhat).mean(-1, keepdims=True)), (dy * xhat).sum(0)
