"""The 8-bit attention path in float64 on the CPU, written from its definitions (include/ptq.h), one row at a time.

Inputs are numpy arrays that hold the stored values exactly; `store` rounds to the storage type where the definition does.
"""
from __future__ import annotations

import numpy as np


def store(x, dtype: str):
    """x rounded to "f32" or "bf16" (nearest, ties to even), as float64."""
    x = np.asarray(x, dtype=np.float32)
    if dtype == "f32":
        return x.astype(np.float64)
    u = x.view(np.uint32).astype(np.uint64)
    u = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16
    return u.astype(np.uint32).view(np.float32).astype(np.float64)


def rmsnorm_quantize(X, dtype="f32", residual=None, gamma=None, eps=1e-5, normalize=True):
    """(codes int64, scales float64, y float64): y = round(x + residual), code = rne(127 u / max|u|) with u = float32(y gamma)."""
    X = np.asarray(X, dtype=np.float64)
    t, n = X.shape
    y = X.copy() if residual is None else store(X.astype(np.float32) + np.asarray(residual, dtype=np.float32), dtype)
    codes, scales = np.zeros((t, n), dtype=np.int64), np.zeros(t)
    for i in range(t):
        u = y[i] if gamma is None else (y[i] * np.asarray(gamma, dtype=np.float64)).astype(np.float32).astype(np.float64)
        if not np.all(np.isfinite(u)):
            scales[i] = np.nan
            continue
        A = np.max(np.abs(u))
        if A == 0:   # codes 0 and scale 0, whatever eps is
            continue
        codes[i] = np.rint(127.0 * u / A)
        scales[i] = A / 127.0
        if normalize:
            scales[i] /= np.sqrt(np.sum(y[i] ** 2) / n + eps)
    return codes, scales, y


def int8_linear(A, a_scales, W, w_scales, bias=None):
    """(sum_k A[i, k] W[j, k]) a_scales[i] w_scales[j] + bias[j]."""
    O = (np.asarray(A, dtype=np.int64) @ np.asarray(W, dtype=np.int64).T).astype(np.float64)
    O = O * np.asarray(a_scales, dtype=np.float64)[:, None] * np.asarray(w_scales, dtype=np.float64)
    return O if bias is None else O + np.asarray(bias, dtype=np.float64)


def quantize_row(x, bits: int):
    """(codes, scale, zero) of one row of the cache."""
    x = np.asarray(x, dtype=np.float64)
    if not np.all(np.isfinite(x)):
        return np.zeros(x.shape, dtype=np.int64), np.nan, 0
    top = 2 ** bits - 1
    lo, hi = min(0.0, x.min()), max(0.0, x.max())
    if np.float32((hi - lo) / top) == 0:
        lo, hi = -1.0, 1.0
        x = np.zeros_like(x)
    scale = float(np.float32((hi - lo) / top))
    zero = int(np.rint(-lo / scale))
    return np.clip(np.rint(x / scale) + zero, 0, top).astype(np.int64), scale, zero


def pack_row(codes, bits: int):
    codes = np.asarray(codes, dtype=np.int64)
    if bits == 8:
        return codes.astype(np.uint8)
    words = []
    for w in codes.reshape(-1, 8):
        words.append(sum(int(c) << (4 * (i // 2) + 16 * (i % 2)) for i, c in enumerate(w)))
    return np.array(words, dtype="<u4").view(np.uint8)


def unpack_row(raw, bits: int):
    """Codes of rows of bytes (any leading dimensions)."""
    raw = np.ascontiguousarray(raw, dtype=np.uint8)
    if bits == 8:
        return raw.astype(np.int64)
    words = raw.view("<u4").astype(np.int64)[..., None]
    i = np.arange(8)
    return ((words >> (4 * (i // 2) + 16 * (i % 2))) & 15).reshape(raw.shape[:-1] + (2 * raw.shape[-1],))


def cache_write(K, V, slots, bits: int, codes, scales, zeros):
    """Writes rows [t, heads, d] into codes [2, pages, heads, page, bytes], scales and zeros, in place."""
    pages, heads, page = codes.shape[1:4]
    for which, X in enumerate((K, V)):
        for i, s in enumerate(np.asarray(slots)):
            if not 0 <= s < pages * page:
                continue
            for h in range(heads):
                c, sc, z = quantize_row(X[i, h], bits)
                codes[which, s // page, h, s % page] = pack_row(c, bits)
                scales[which, s // page, h, s % page] = sc
                zeros[which, s // page, h, s % page] = z


def cache_rows(codes, scales, zeros, bits: int, table, length: int, which: int):
    """What the cache holds of one sequence: ([length, heads, d] float64, [length] whether the page is there)."""
    pages, _, page = codes.shape[1:4]
    i = np.arange(length)
    p = np.full(length, -1, dtype=np.int64)
    listed = i // page < len(table)
    p[listed] = np.asarray(table, dtype=np.int64)[i[listed] // page]
    there = (p >= 0) & (p < pages)
    p = np.where(there, p, 0)
    X = unpack_row(codes[which][p, :, i % page], bits) - zeros[which][p, :, i % page].astype(np.int64)[..., None]
    X = scales[which][p, :, i % page].astype(np.float64)[..., None] * X
    X[~there] = 0.0
    return X, there


def attention(Q, cu_q, codes, scales, zeros, bits: int, table, kv_lens, softmax_scale: float, causal=True, window=0, spread=False):
    """Query i of a sequence of `new` queries and `length` keys stands at place length - new + i; it sees key j if j < length,
    j's page is there, and (causal) j <= place, (window > 0) j > place - window.  No key: zeros.
    spread: also sum p |v| / sum p and the largest softmax_scale sum |q| |k| of each (token, head), for error bounds."""
    Q = np.asarray(Q, dtype=np.float64)
    group = Q.shape[1] // codes.shape[2]
    O, size, reach = np.zeros(Q.shape), np.zeros(Q.shape), np.zeros(Q.shape[:2])
    for s, length in enumerate(kv_lens):
        a, b, length = int(cu_q[s]), int(cu_q[s + 1]), int(length)
        if a == b:
            continue
        K, there = cache_rows(codes, scales, zeros, bits, table[s], length, 0)
        V, _ = cache_rows(codes, scales, zeros, bits, table[s], length, 1)
        place, j = length - (b - a) + np.arange(b - a)[:, None], np.arange(length)[None]
        sees = np.broadcast_to(there, (b - a, length)).copy()
        if causal:
            sees &= j <= place
        if window:
            sees &= j > place - window
        some = sees.any(1)
        if not some.any():
            continue
        for h in range(Q.shape[1]):
            k, v = K[:, h // group], V[:, h // group]
            for rows in np.array_split(np.nonzero(some)[0], max(1, int(some.sum()) * length // 4000000)):
                # a key that a query does not see has no part in it, whatever it holds
                with np.errstate(invalid="ignore"):
                    x = np.where(sees[rows], softmax_scale * (Q[a + rows, h] @ np.where(np.isnan(k), 0.0, k).T), -np.inf)
                x[sees[rows] & np.isnan(k).any(1)] = np.nan
                p = np.exp(x - x.max(1, keepdims=True))
                lost = (sees[rows] & np.isnan(v).any(1)).any(1)
                O[a + rows, h] = p @ np.where(np.isnan(v), 0.0, v) / p.sum(1, keepdims=True)
                O[a + rows[lost], h] = np.nan
                if spread:
                    size[a + rows, h] = p @ np.abs(np.where(np.isnan(v), 0.0, v)) / p.sum(1, keepdims=True)
                    r = abs(softmax_scale) * (np.abs(Q[a + rows, h]) @ np.abs(np.where(np.isnan(k), 0.0, k)).T)
                    reach[a + rows, h] = np.where(sees[rows], r, 0).max(1)
    return (O, size, reach) if spread else O


def rotary(X, positions, freq, scale=1.0, interleaved=False, dtype="f32"):
    """X (tokens x heads x d) with its first 2 len(freq) channels turned pair by pair; angles in extended precision (64 bits of fraction)."""
    X = np.asarray(X, dtype=np.float64)
    half = len(freq)
    angle = np.outer(np.asarray(positions).astype(np.longdouble), np.asarray(freq, dtype=np.float64).astype(np.longdouble))
    cos, sin = (scale * np.cos(angle)).astype(np.float64), (scale * np.sin(angle)).astype(np.float64)
    Y = X.copy()
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        Y[:, :, a] = X[:, :, a] * cos[:, j, None] - X[:, :, b] * sin[:, j, None]
        Y[:, :, b] = X[:, :, a] * sin[:, j, None] + X[:, :, b] * cos[:, j, None]
    return store(Y, dtype)
