"""Dropout from a counter-based generator, LayerNorm behind dropout and a residual sum, and attention with a learned, bucketed
relative position bias, forward and backward: the definitions in numpy float64 and whole numbers (TEST INFRASTRUCTURE ONLY).

The generator is Philox4x32-10 (Salmon, Moraes, Dror and Shaw, 2011), pinned by its published test vectors.  The backward passes
are pinned by central differences (tests/test_oracle_training_ops.py).
"""
from __future__ import annotations

import numpy as np

_M = 0xFFFFFFFF


# ---------------------------------------------------------------- generator and dropout
def philox4x32(counter, key, rounds=10):
    """Four 32-bit words for a counter of four and a key of two, Python integers or arrays of them (uint64)."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k = [int(w) & _M for w in key]
    sh, m = np.uint64(32), np.uint64(_M)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> sh) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> sh) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & _M, (k[1] + 0xBB67AE85) & _M]
    return c


def dropout_threshold(p):
    return int(np.rint(np.float64(np.float32(p)) * 65536))


def keep_mask(rows, cols, p, seed, step, site, first_row=0):
    """[rows, cols] of truth values."""
    col, row = np.meshgrid(np.arange(cols, dtype=np.uint64), (np.arange(rows, dtype=np.uint64) + np.uint64(first_row)) & np.uint64(_M))
    w = np.stack(philox4x32((col >> np.uint64(3), row, np.uint64(site & _M), np.uint64(step & _M)), (seed & _M, (seed >> 32) & _M)))
    j = (col & np.uint64(7)).astype(np.int64)
    word = np.take_along_axis(w, (j // 2)[None], 0)[0]
    return ((word >> (np.uint64(16) * (col & np.uint64(1)))) & np.uint64(0xFFFF)).astype(np.int64) >= dropout_threshold(p)


def dropout(x, keep, p):
    t = dropout_threshold(p)
    up = 65536.0 / (65536 - t) if t < 65536 else 0.0
    return np.where(keep, x * up, 0.0) if t else x


# ---------------------------------------------------------------- LayerNorm
def layernorm_fwd(s, gamma, beta, eps):
    mean = s.mean(-1)
    rstd = 1.0 / np.sqrt(((s - mean[..., None]) ** 2).mean(-1) + eps)
    xh = (s - mean[..., None]) * rstd[..., None]
    return (xh if gamma is None else xh * gamma + beta), mean, rstd


def layernorm_bwd(dy, s, mean, rstd, gamma):
    """Gradients of s, gamma and beta."""
    xh = (s - mean[..., None]) * rstd[..., None]
    g = dy if gamma is None else dy * gamma
    ds = rstd[..., None] * (g - g.mean(-1, keepdims=True) - xh * (g * xh).mean(-1, keepdims=True))
    return ds, (dy * xh).sum(0), dy.sum(0)


# ---------------------------------------------------------------- relative position bias
def bucket(distance, n_buckets, max_distance, bidirectional):
    """Bucket of a distance key - query.  The buckets of one direction: half of them for one distance each, the others growing with the
    logarithm, bucket half + k from the least n with (n / half)^(rest) >= (max_distance / half)^k on, the last without end.  Both directions
    share the buckets out where they count (the second half for keys behind the query); else keys behind the query are in bucket 0."""
    nb = n_buckets // 2 if bidirectional else n_buckets
    n = abs(distance) if bidirectional else max(-distance, 0)
    side = nb if bidirectional and distance > 0 else 0
    half = nb // 2
    if n < half:
        return side + n
    rest = nb - half
    k = 0
    while k + 1 < rest and n ** rest * half ** (k + 1) >= max_distance ** (k + 1) * half ** rest:
        k += 1
    return side + half + k


def buckets(nq, nk, query0, n_buckets, max_distance, bidirectional):
    lo = -(nq - 1) - query0
    by = np.array([bucket(lo + c, n_buckets, max_distance, bidirectional) for c in range(nq + nk - 1)])
    return by[np.arange(nk)[None] - np.arange(nq)[:, None] + nq - 1]


# ---------------------------------------------------------------- attention, [B, H, N, d]
def _logits(q, k, scale, table, bk, causal, query0, key_len):
    s = scale * (q @ np.swapaxes(k, -1, -2))
    if table is not None:
        s = s + np.moveaxis(np.where(table <= -65536.0, -np.inf, table)[bk], -1, 0)[None]      # entries from there on mask their pairs
    nq, nk = s.shape[-2:]
    j = np.arange(nk)
    if causal:
        s = np.where((j[None] <= np.arange(nq)[:, None] + query0)[None, None], s, -np.inf)
    if key_len is not None:
        s = np.where((j[None] < np.asarray(key_len)[:, None])[:, None, None], s, -np.inf)
    return s


def attention_relbias_fwd(q, k, v, scale, table, bk, causal=False, query0=0, key_len=None):
    """O and the logarithm of the softmax sums; a query that sees no key has zeros and -infinity.  Values of keys that nobody sees
    (beyond a sample's key length) must be finite here."""
    s = _logits(q, k, scale, table, bk, causal, query0, key_len)
    m = s.max(-1, keepdims=True)
    e = np.exp(s - np.where(np.isneginf(m), 0.0, m))
    z = e.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (m + np.log(z))[..., 0]
    return (e / np.where(z == 0, 1.0, z)) @ v, lse


def attention_relbias_bwd(q, k, v, o, lse, do, scale, table, bk, causal=False, query0=0, key_len=None):
    """Gradients of q, k, v and the table."""
    s = _logits(q, k, scale, table, bk, causal, query0, key_len)
    p = np.exp(s - np.where(np.isneginf(lse), 0.0, lse)[..., None])
    ds = p * (do @ np.swapaxes(v, -1, -2) - (do * o).sum(-1, keepdims=True))
    per_pair = ds.sum(0)
    dt = np.zeros_like(table)
    for h in range(table.shape[1]):
        dt[:, h] = np.bincount(bk.ravel(), per_pair[h].ravel(), table.shape[0])
    return scale * (ds @ k), scale * (np.swapaxes(ds, -1, -2) @ q), np.swapaxes(p, -1, -2) @ do, dt
