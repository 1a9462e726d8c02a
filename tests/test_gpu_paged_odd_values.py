"""Values that are not finite, at the masks' edges of many items that one CTA of the kernel for many rows takes one after
another: each of them shows in the rows that see it, and in nothing else."""
import numpy as np
import pytest

from tests.paged_util import Paged, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,d", [(8, 64), (8, 128), (7, 128), (4, 256)])
@pytest.mark.parametrize("sizes", [(20, 5), (30, 17, 2), (24,), (3, 40)])
@pytest.mark.parametrize("old", [0, 150])
def test_every_item_has_its_own(cuda_device, H, d, sizes, old):
    """Items of one and of two row tiles in turn (rows of 128: 16, 18 or 32 queries)."""
    R = 900
    new = [sizes[r % len(sizes)] for r in range(R)]
    s = Paged(new, [n + old for n in new], H, 1, d, 16, seed=d + len(sizes))
    s.many = True
    clean = host(s.run())
    want, rng = clean.copy(), np.random.default_rng(5)
    for r in range(R):
        if rng.random() < 0.3:
            continue  # (and some without)
        at, col = int(rng.integers(0, new[r])), int(rng.integers(0, d))
        pg, place = s.at(r, old + at)
        s.v[pg, place, 0, col] = [np.nan, np.inf, -np.inf][r % 3]
        rows = slice(s.q_start[r] + at, s.q_start[r + 1])
        want.reshape(-1, H, d)[rows, :, col] = s.v[pg, place, 0, col]
    for _ in range(4):
        out = host(s.run())
        assert np.array_equal(out, want, equal_nan=True)
