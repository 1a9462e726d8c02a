"""Capped scores cap * tanh(s / cap) for caps of every size: a cap far above the scores leaves them as they are, to fp32's
precision of the score and not of the cap; one far below them makes all scores of a sign alike."""
import numpy as np
import pytest

from oracle.layer import U32, U_BF16
from tests.paged_util import Paged, check, host

pytestmark = pytest.mark.gpu


def _reference(s, cap, weight_error):
    """(ref, bound) of causal queries in 64 bits. Bound: the dot product and its scaling are within 2 (d + 2) u |scale| sum |q k|
    of exact; the capped score z within 2^-20 |z| more, as it is formed with a few fp32 operations and hardware functions of
    2^-22; a weight within a relative 2^-10 + weight_error; sums as in the oracle; the bf16 store 2^-8."""
    G, d, cap = s.H // s.Hk, s.d, float(np.float32(cap))
    ref, bound = np.zeros((s.T, s.H * d)), np.zeros((s.T, s.H * d))
    for r, (n, L) in enumerate(zip(s.new, s.kv)):
        pages, place = s.table[r][np.arange(L) // s.page], np.arange(L) % s.page
        for i in range(n):
            t, hi = s.q_start[r] + i, L - n + i + 1
            for h in range(s.H):
                q = s.q[t, h * d:(h + 1) * d].astype(np.float64)
                k, v = (c[pages[:hi], place[:hi], h // G].astype(np.float64) for c in (s.k, s.v))
                x = s.scale * (k @ q)
                z = cap * np.tanh(x / cap)
                w = np.exp(z - z.max())
                p = w / w.sum()
                rho = 2 * (d + 2) * U32 * abs(s.scale) * (np.abs(k) @ np.abs(q)).max() + 2.0 ** -20 * np.abs(z).max() + 2.0 ** -10 + weight_error
                err = (2.2 * rho + 4.0 * (hi + 8) * U32) * (p @ np.abs(v))
                at = slice(h * d, (h + 1) * d)
                ref[t, at] = p @ v
                bound[t, at] = err + U_BF16 * (np.abs(ref[t, at]) + err) + 1e-38
    return ref, bound


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("new,kv,H,Hk,d", [([1], [700], 8, 1, 128), ([6, 2], [90, 300], 4, 2, 64), ([1], [300], 4, 1, 256), ([40], [260], 7, 1, 64)])
@pytest.mark.parametrize("cap", [1e-42, 1e-30, 1e-3, 0.7, 8.0, 1e3, 1e5, 1e7, 1e12, 1e25, 3e38])
def test_caps_of_every_size(cuda_device, cap, new, kv, H, Hk, d, many):
    s = Paged(new, kv, H, Hk, d, 16, seed=d + H, gain=4.0)
    s.many = many
    check(host(s.run(cap=cap))[:s.T], *_reference(s, cap, 2.0 ** -8 if many or max(new) * H > 16 * Hk else 0.0), f"cap={cap}")
