"""Oracle for the 8-bit paged key/value cache (TEST INFRASTRUCTURE ONLY; same import rules as the rest of ``oracle``): the
e4m3 codes, the blocks' exponents, the store's rule and the turns of the rotation, written out plainly in numpy from the format's
definition. Attention is that of the bf16 cache over the codes' values.
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

from .layer import U32, U_BF16

BLOCK = 16
EXP_MOST = 48
CODE_MOST = 448.0
U_E4M3 = 2.0 ** -4     # half a step of a normal code, relative to the value
NAN_CODE = 0x7F


def e4m3_values():
    """What the 256 codes stand for."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, (c & 7).astype(np.float64)
    x = np.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7.0), m / 8 * 2.0 ** -6)
    x[(c & 0x7F) == NAN_CODE] = np.nan
    return np.where(c & 0x80, -x, x)


def e4m3_codes(x):
    """Nearest codes of values of at most 448 in magnitude, ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    table = e4m3_values()[:NAN_CODE]                                     # rising
    a = np.abs(x)
    hi = np.clip(np.searchsorted(table, a), 0, NAN_CODE - 1)
    lo = np.maximum(hi - 1, 0)
    down, up = a - table[lo], table[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def exponent_of(byte):
    return np.clip(np.asarray(byte).astype(np.int64) - 127, -EXP_MOST, EXP_MOST)


def need_of(top):
    """The least exponent in -48..48 under which `top` is at most 448."""
    for e in range(-EXP_MOST, EXP_MOST):
        if top <= CODE_MOST * 2.0 ** e:
            return e
    return EXP_MOST


def paged8_values(codes, exps):
    """fp64 values of a cache [n_pages][page_size][Hk][d] with exponents [n_pages][page_size / 16][Hk]."""
    x = e4m3_values()[codes]
    return x * 2.0 ** np.repeat(exponent_of(exps), BLOCK, axis=1)[..., None]


def paged8_encode(x):
    """Codes and exponent bytes of a whole cache of values, every block by itself."""
    n, page, Hk, d = x.shape
    blocks = np.asarray(x, dtype=np.float64).reshape(n, page // BLOCK, BLOCK, Hk, d)
    top = np.abs(np.where(np.isfinite(blocks), blocks, 0)).max(axis=(2, 4))
    e = np.vectorize(need_of, otypes=[np.int64])(top)
    y = blocks * 2.0 ** -e[:, :, None, :, None]
    codes = np.where(np.isfinite(blocks), e4m3_codes(np.where(np.isfinite(y), y, 0)), NAN_CODE)
    return codes.astype(np.uint8).reshape(x.shape), (e + 127).astype(np.uint8)


def paged8_store_reference(rows, codes, exps, slots):
    """Rows [T][Hk][d] (fp64) into copies of a cache's codes and exponents, block by block. Returns (codes, exps)."""
    codes, exps = codes.copy(), exps.copy()
    n_pages, page, Hk, d = codes.shape
    value = e4m3_values()
    limit = CODE_MOST * 2.0 ** EXP_MOST
    blocks = {}
    for t, s in enumerate(slots):
        if 0 <= s < n_pages * page:
            blocks.setdefault(int(s) // BLOCK, {})[int(s) % BLOCK] = t
    for b, places in blocks.items():
        pg, in_page = b * BLOCK // page, b * BLOCK % page
        for h in range(Hk):
            new = {i: np.where(np.abs(rows[t, h]) <= limit, rows[t, h], np.nan) for i, t in places.items()}
            tops = [np.abs(x[np.isfinite(x)]).max(initial=0.0) for x in new.values()]
            e, was = need_of(max(tops)), int(exponent_of(exps[pg, in_page // BLOCK, h]))
            fresh = 0 in places
            if not fresh:
                e = max(e, was)
            exps[pg, in_page // BLOCK, h] = e + 127
            for i in range(BLOCK):
                at = (pg, in_page + i, h)
                if i in new:
                    x = new[i]
                elif fresh:
                    x = np.zeros(d)
                elif e == was:
                    continue
                else:
                    x = value[codes[at]] * 2.0 ** was
                ok = np.isfinite(x)
                c = e4m3_codes(np.where(ok, x, 0) * 2.0 ** -e)
                if i in new or fresh:
                    codes[at] = np.where(ok, c, NAN_CODE)
                else:
                    codes[at] = np.where(ok, c, codes[at])
    return codes, exps


def rotary_turns_reference(rot_dim: int, base: float, stretch: float = 1.0, original: float = 0.0, low: float = 1.0, high: float = 32.0):
    """Turns per position of each pair, in units of 2^-64, as exact fractions of the fp64 formula's value."""
    out = []
    for i in range(rot_dim // 2):
        f = math.pow(base, -2.0 * i / rot_dim) / (2.0 * math.pi)
        if stretch > 1.0:
            keep = min(1.0, max(0.0, (original * f - low) / (high - low))) if original > 0 else 0.0
            f = f * (keep + (1.0 - keep) / stretch)
        out.append(Fraction(f) % 1 * 2 ** 64)
    return out


def norm_turn_reference(x, n_heads: int, head_dim: int, gamma, eps: float, positions, axis_of_pair, turns, neighbours: bool = False,
                        factor: float = 1.0):
    """x: bf16 values [T][H * d]; positions: [axes][T] integers; turns: [rot_dim / 2] integers. Returns (y, err), [T][H][d]: the
    fp64 value and a bound on any fp32 implementation's, before the last rounding.

    Bound: as for the bf16 cache, with cosine and sine within 2^-19 at every position (an allowance above the contract's 1e-6:
    the angle is formed in whole numbers), times the factor's magnitude and one more rounding for it."""
    x = np.asarray(x, dtype=np.float64)
    T = x.shape[0]
    half = len(turns)
    y = x.reshape(T, n_heads, head_dim).copy()
    e = 0.0
    if gamma is not None:
        y = y / np.sqrt(np.mean(y * y, axis=2, keepdims=True) + float(np.float32(eps))) * np.asarray(gamma, dtype=np.float64)
        e = (head_dim + 16) * U32
    out, err = y.copy(), e * np.abs(y)
    if half:
        factor = float(np.float32(factor))
        pos = np.asarray(positions).astype(object)[np.asarray(axis_of_pair)].T                       # [T][half]
        turn = pos * np.array([int(t) for t in turns], dtype=object)[None]
        frac = np.vectorize(lambda t: float(Fraction(t % 2 ** 64, 2 ** 64)), otypes=[np.float64])(turn) if T else np.zeros((0, half))
        c, s = factor * np.cos(2 * np.pi * frac)[:, None], factor * np.sin(2 * np.pi * frac)[:, None]
        a_at = np.arange(half) * (2 if neighbours else 1)
        b_at = a_at + (1 if neighbours else half)
        a, b = y[..., a_at], y[..., b_at]
        out[..., a_at], out[..., b_at] = a * c - b * s, b * c + a * s
        mag = (np.abs(a) + np.abs(b)) * abs(factor)
        err[..., a_at] = err[..., b_at] = (e + 2.0 ** -19 + 6 * U32) * mag
    return out, err


def bf16_bound(y, err):
    """The bound of a value within `err` of y after one rounding to bf16."""
    return err + U_BF16 * (np.abs(y) + err) + 1e-38
