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
        if A > 0:
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
    raw = np.ascontiguousarray(raw, dtype=np.uint8)
    if bits == 8:
        return raw.astype(np.int64)
    return np.array([(int(w) >> (4 * (i // 2) + 16 * (i % 2))) & 15 for w in raw.view("<u4") for i in range(8)], dtype=np.int64)


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
    pages, heads, page = codes.shape[1:4]
    d = codes.shape[4] * 8 // bits
    X, there = np.zeros((length, heads, d)), np.zeros(length, dtype=bool)
    for i in range(length):
        p = int(table[i // page]) if i // page < len(table) else -1
        if not 0 <= p < pages:
            continue
        there[i] = True
        for h in range(heads):
            at = (which, p, h, i % page)
            X[i, h] = float(scales[at]) * (unpack_row(codes[at], bits) - int(zeros[at]))
    return X, there


def attention(Q, cu_q, codes, scales, zeros, bits: int, table, kv_lens, softmax_scale: float, causal=True, window=0):
    """Query i of a sequence of `new` queries and `length` keys stands at place length - new + i; it sees key j if j < length,
    j's page is there, and (causal) j <= place, (window > 0) j > place - window.  No key: zeros."""
    Q = np.asarray(Q, dtype=np.float64)
    hq, hkv = Q.shape[1], codes.shape[2]
    O = np.zeros(Q.shape)
    for s, length in enumerate(kv_lens):
        a, b = int(cu_q[s]), int(cu_q[s + 1])
        K, there = cache_rows(codes, scales, zeros, bits, table[s], int(length), 0)
        V, _ = cache_rows(codes, scales, zeros, bits, table[s], int(length), 1)
        j = np.arange(int(length))
        for i in range(b - a):
            place = int(length) - (b - a) + i
            sees = there.copy()
            if causal:
                sees &= j <= place
            if window:
                sees &= j > place - window
            if not sees.any():
                continue
            for h in range(hq):
                g = h // (hq // hkv)
                x = softmax_scale * (K[sees, g] @ Q[a + i, h])
                p = np.exp(x - x.max())
                O[a + i, h] = p @ V[sees, g] / p.sum()
    return O
