"""Products q.k beyond fp32's range under a cap: one below it is a score of -cap and has its part in the softmax, as one above it is
a score of cap, in both kernels, beside hidden keys and ordinary ones."""
import numpy as np
import pytest

from tests.paged_util import host
from tests.paged8_util import F16_WEIGHT, Paged8

pytestmark = pytest.mark.gpu


def expected(s, cap, sign, lo, hi):
    """Outputs of one head of a request's queries whose scores are cap * sign[key], and their bound: a score within 2^-20 cap, a
    weight within 2^-10 and its rounding to f16, fp32 sums, one bf16 rounding."""
    v = s.v[s.table[0][np.arange(s.kv[0]) // s.page], np.arange(s.kv[0]) % s.page, 0]
    ref, bound = [], []
    for a, b in zip(lo, hi):
        w = np.exp(cap * (sign[a:b] - sign[a:b].max()))
        w /= w.sum()
        o, mag = w @ v[a:b], w @ np.abs(v[a:b])
        err = (2.2 * (2.0 ** -20 * cap + 2.0 ** -10 + F16_WEIGHT) + 4 * (b - a + 8) * 2.0 ** -24) * mag
        ref.append(o)
        bound.append(err + 2.0 ** -8 * (np.abs(o) + err))
    return np.array(ref)[:, None], np.array(bound)[:, None]


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,kv", [(1, 300), (1, 3000), (60, 500), (150, 150)])
@pytest.mark.parametrize("cap", [2.0, 50.0, 500.0])
@pytest.mark.parametrize("signs", ["low", "low and ordinary", "all"])
def test_products_beyond_the_range(cuda_device, signs, cap, new, kv, d, many):
    s = Paged8([new], [kv], 2, 1, d, 32, seed=kv + d)
    s.many = many
    s.scale = 1.0
    s.q = np.full_like(s.q, 2.0 ** 100)
    sign = s.rng.choice({"low": [-1], "low and ordinary": [-1, -1, 0], "all": [-1, 0, 1]}[signs], kv).astype(float)
    s.k[:] = 0.0
    for pos in range(kv):
        s.k[s.at(0, pos)] = sign[pos] * 2.0 ** 50
    s.garble_unused()
    at = np.arange(kv - new, kv)
    for mask, lo, hi in (({}, 0 * at, at + 1), ({"prefix": [kv]}, 0 * at, 0 * at + kv), ({"window": 70}, np.maximum(at - 69, 0), at + 1)):
        out = host(s.run(cap=cap, **mask))[:new].reshape(new, 2, d)
        ref, bound = expected(s, cap, sign, lo, hi)
        assert (np.abs(out - ref) <= bound).all(), (mask, np.abs(out - ref).max())
