"""Oracle for the paged key/value cache (TEST INFRASTRUCTURE ONLY; same import rules as the
rest of ``oracle``): a step's block table, slots and positions, per-head norm with rotation and
cache write, and attention over the cache, written out plainly in numpy.

The floating-point functions return the fp64 reference and a per-element bound on
|GPU - reference| that any correct fp32 implementation with a final bf16 rounding meets; the
derivations are in the docstrings and build on those of the layer steps.
"""
from __future__ import annotations

import numpy as np

from .layer import U32, U_BF16


def paged_slots_reference(cached, added, free_pages, used: int, page_size: int, table, n_tokens: int):
    """Whole numbers, token by token. Returns (table, q_start, kv_len, slots, positions, used_out)."""
    cached = [max(0, int(c)) for c in cached]
    added = [max(0, int(a)) for a in added]
    table = np.array(table, dtype=np.int64)
    R, max_pages = table.shape
    slots = np.full(n_tokens, -1, dtype=np.int64)
    positions = np.zeros(n_tokens, dtype=np.int64)
    q_start = np.zeros(R + 1, dtype=np.int64)
    at = 0
    for r in range(R):
        q_start[r] = at
        have = min(-(-cached[r] // page_size), max_pages)
        want = min(-(-(cached[r] + added[r]) // page_size), max_pages)
        taken = [int(free_pages[used + i]) if 0 <= used + i < len(free_pages) else -1 for i in range(want - have)]
        for i in range(added[r]):
            t, pos = at + i, cached[r] + i
            if t >= n_tokens:
                break
            positions[t] = pos
            pg = pos // page_size
            if pg >= max_pages:
                continue
            if pg >= have:
                table[r, pg] = taken[pg - have]
            if table[r, pg] >= 0:
                slots[t] = table[r, pg] * page_size + pos % page_size
        used += want - have
        at += added[r]
    q_start[R] = at
    kv_len = np.array([c + a for c, a in zip(cached, added)], dtype=np.int64)
    return table, q_start, kv_len, slots, positions, used


def qk_norm_rope_reference(x, n_heads: int, head_dim: int, gamma, eps: float, positions, axis_of_pair,
                           rot_dim: int, base: float):
    """x: bf16 values [T][H*d]; gamma: [d] or None; positions: [axes][T]; axis_of_pair: [rot_dim / 2].
    Returns (ref, bound), [T][H*d].

    Bound: the norm's fp32 value is within e = (d + 16) u of exact (as for RMSNorm over the width; 0
    without gamma); cosine and sine are within 2^-19 of exact below 2^24 (an allowance above the
    contract's 1e-6), 1e-5 beyond, and the rotation adds two products and one sum, so its value is
    within (e + t + 4 u) (|y_a| + |y_b|); the bf16 store adds 2^-8 of the value."""
    x = np.asarray(x, dtype=np.float64)
    T = x.shape[0]
    half = rot_dim // 2
    y = x.reshape(T, n_heads, head_dim).copy()
    e = 0.0
    if gamma is not None:
        y = y / np.sqrt(np.mean(y * y, axis=2, keepdims=True) + float(np.float32(eps))) * np.asarray(gamma, dtype=np.float64)
        e = (head_dim + 16) * U32
    ref, mag = y.copy(), np.abs(y)
    t = 2.0 ** -19 if not np.size(positions) or np.abs(positions).max() < 2 ** 24 else 1e-5
    if half:
        i = np.arange(half, dtype=np.float64)
        freq = float(np.float32(base)) ** (-2.0 * i / rot_dim)
        pos = np.asarray(positions, dtype=np.float64)[np.asarray(axis_of_pair)].T      # [T][half]
        c, s = np.cos(pos * freq)[:, None], np.sin(pos * freq)[:, None]
        a, b = y[..., :half], y[..., half:rot_dim]
        ref[..., :half] = a * c - b * s
        ref[..., half:rot_dim] = b * c + a * s
        mag[..., :half] = mag[..., half:rot_dim] = np.abs(a) + np.abs(b)
        err = (e + t + 4 * U32) * mag
        err[..., rot_dim:] = e * mag[..., rot_dim:]
    else:
        err = e * mag
    bound = err + U_BF16 * (np.abs(ref) + err) + 1e-38
    return ref.reshape(T, -1), bound.reshape(T, -1)


def paged_attention_reference(Q, k_cache, v_cache, table, q_start, kv_len, n_heads: int, scale: float, prefix=None,
                              cap: float = 0.0, window: int = 0, weight_error: float = 0.0):
    """Q: [T][H*d]; caches: [n_pages][page_size][Hk][d]; table: [R][max_pages]. Query by query, only the keys it
    sees. Returns (ref, bound), [T][H*d]; rows of no request and of queries without a key are 0.

    Bound, per query and head with n visible keys: as for the contiguous attention, each score is within Delta = 2 (d + 2)
    u |scale| max_j sum_i |q_i k_ji| of exact, plus 2^-20 cap when capped (tanh within 2^-21 of exact, slope at
    most 1); each unnormalised weight is within a relative 2^-10 of exp of the computed score, plus
    `weight_error` where the weights of the value product are rounded further (2^-8 for one bf16); so
    |o error| <= (2.2 rho + 4 (n + 8) u) sum_j p_j |v_j|, and the bf16 store adds 2^-8 |o|."""
    Q = np.asarray(Q, dtype=np.float64)
    n_pages, page_size, Hk, d = k_cache.shape
    T = Q.shape[0]
    G = n_heads // Hk
    ref = np.zeros((T, n_heads * d))
    bound = np.full((T, n_heads * d), 1e-38)
    for r in range(len(kv_len)):
        a, b = min(int(q_start[r]), T), min(int(q_start[r + 1]), T)
        m, L = b - a, min(int(kv_len[r]), table.shape[1] * page_size)
        f = min(int(prefix[r]), L) if prefix is not None else 0
        keys = np.arange(max(L, 0))
        pages = np.asarray(table[r])[keys // page_size].astype(np.int64) if L > 0 else keys
        ok = (pages >= 0) & (pages < n_pages)
        at = np.where(ok, pages, 0)
        K = np.where(ok[:, None, None], k_cache[at, keys % page_size], 0.0)            # [L][Hk][d]
        V = np.where(ok[:, None, None], v_cache[at, keys % page_size], 0.0)
        for i in range(m):
            p = L - m + i
            lo, hi = (max(0, p - window + 1) if window > 0 else 0), min(L, max(p + 1, f))
            if hi <= lo:
                continue
            for g in range(Hk):
                q = Q[a + i, g * G * d:(g + 1) * G * d].reshape(G, d)
                k, v = K[lo:hi, g], V[lo:hi, g]
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (q @ k.T)
                    if cap > 0:
                        s = cap * np.tanh(s / cap)
                    w = np.exp(s - s.max(axis=1, keepdims=True))
                    pr = w / w.sum(axis=1, keepdims=True)
                    o = pr @ v
                    rho = (2 * (d + 2) * U32 * abs(scale) * (np.abs(q) @ np.abs(k).T).max(axis=1, keepdims=True)
                           + (2.0 ** -20 * cap if cap > 0 else 0.0) + 2.0 ** -10 + weight_error)
                    err = (2.2 * rho + 4.0 * (hi - lo + 8) * U32) * (pr @ np.abs(v))
                    ref[a + i, g * G * d:(g + 1) * G * d] = o.reshape(-1)
                    bound[a + i, g * G * d:(g + 1) * G * d] = (err + U_BF16 * (np.abs(o) + err) + 1e-38).reshape(-1)
    return ref, bound
