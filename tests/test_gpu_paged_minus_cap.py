"""Scores of -infinity under a cap are scores of -cap: they have their part in the softmax."""
import numpy as np
import pytest

from oracle.layer import U32
from tests.paged_util import Paged, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("new,kv", [(1, 300), (1, 30000), (60, 500)])
@pytest.mark.parametrize("cap", [5.0, 50.0, 500.0])
def test_all_scores_alike_give_the_mean_of_the_values(cuda_device, cap, new, kv, many):
    """Bound: equal weights, each 2^0 once its row's maximum is taken off; fp32 sums, one bf16 rounding."""
    s = Paged([new], [kv], 2, 1, 128, 64, seed=kv)
    s.many = many
    s.q = np.abs(s.q) + 0.5
    s.k[:] = -np.inf
    v = s.v[s.table[0][np.arange(kv) // s.page], np.arange(kv) % s.page, 0].astype(np.float64)
    n = np.arange(kv - new + 1, kv + 1)[:, None]
    mean, mag = np.cumsum(v, axis=0)[kv - new:] / n, np.cumsum(np.abs(v), axis=0)[kv - new:] / n
    out = host(s.run(cap=cap))[:new].reshape(new, 2, 128)
    bound = (2.0 ** -8 + 4 * (kv + 8) * U32) * mag + 2.0 ** -8 * np.abs(mean)
    assert (np.abs(out - mean[:, None]) <= bound[:, None]).all()
