"""Large queries under a large scale: the factor of a row, the scale and a block's power multiply to a number in fp32's range, also
where the first two by themselves do not."""
import numpy as np
import pytest

from tests.paged_util import host
from tests.paged8_util import Paged8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 150])
@pytest.mark.parametrize("q,scale", [(2.0 ** 100, 2.0 ** 46), (2.0 ** 120, -2.0 ** 30), (2.0 ** -60, 2.0 ** 50), (2.0 ** 127, 2.0 ** -60), (2.0 ** -120, 1.0)])
def test_the_order_of_far_apart_scores(cuda_device, q, scale, new, d, many):
    """One key's score exceeds the others' by powers of two, so it has all the weight, although its code is the least of its block;
    where all scores are below 2^-30, the output is the mean, within twice that and the roundings."""
    s = Paged8([new], [new + 60], 2, 1, d, 16, seed=d)
    s.many = many
    s.scale = scale
    s.q = np.zeros_like(s.q)
    s.q[:, 0::d] = q
    s.k[:] = 0.0
    sign = np.sign(scale)
    best, next_best = s.at(0, 5), s.at(0, 40)
    s.k[best][0, :2] = sign * 2.0 ** -29, 2.0 ** -12       # the least code of a block with the power 2^-20
    s.k[next_best][0, 0] = sign * 2.0 ** -40               # a large code under 2^-48
    s.encode()
    assert s.k[best][0, 0] == sign * 2.0 ** -29 and s.k[next_best][0, 0] == sign * 2.0 ** -40
    out = host(s.run()).reshape(new, 2, d)
    assert np.isfinite(out).all()
    v = s.v[s.table[0][np.arange(new + 60) // 16], np.arange(new + 60) % 16, 0]
    if q * abs(scale) * 2.0 ** -29 > 2.0 ** 20:
        assert np.array_equal(out, np.broadcast_to(v[5], out.shape))
    else:
        assert q * abs(scale) * 2.0 ** -29 < 2.0 ** -30
        n = np.arange(61, new + 61)[:, None]
        mean, mag = np.cumsum(v, axis=0)[60:] / n, np.cumsum(np.abs(v), axis=0)[60:] / n
        bound = (2.0 ** -28 + 2.2 * (2.0 ** -10 + 2.0 ** -11) + 4 * (new + 68) * 2.0 ** -24) * mag + 2.0 ** -8 * np.abs(mean) * 1.01
        assert (np.abs(out - mean[:, None]) <= bound[:, None]).all()
