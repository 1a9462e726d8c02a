"""Capped scores on the kernel for many rows: a query's bits are its own. Neither what an earlier launch left in
shared memory nor another request's queries decides how its scores are computed."""
import numpy as np
import pytest
import torch

import paper_2607_02501_gb300 as emb
from tests.paged_util import Paged, dev_i32

pytestmark = pytest.mark.gpu
CAP = 50.0


def _fill(d, q_value):
    """A call that leaves queries of that value in every row of every SM's row tiles."""
    n, H = 40000 // d, 8
    q = torch.full((4 * n, H * d), q_value, dtype=torch.bfloat16, device="cuda")
    cache = torch.ones(2, 16, 1, d, dtype=torch.bfloat16, device="cuda")
    O = torch.empty_like(q)
    emb.emb_paged_attention(q, cache, cache, dev_i32([[0, 1]] * 4), dev_i32(np.arange(5) * n), dev_i32([32] * 4), O, d ** -0.5, n,
                            emb.paged_workspace(), cap=CAP)


@pytest.mark.parametrize("H,Hk,d", [(14, 2, 64), (3, 1, 128), (10, 2, 64), (6, 1, 128), (7, 1, 256), (28, 4, 128)])
@pytest.mark.parametrize("new", [[300, 170], [20, 9, 33]])
def test_bits_do_not_depend_on_what_ran_before(cuda_device, H, Hk, d, new):
    """Heads per key/value head that leave rows of a 128-row tile unfilled."""
    s = Paged(new, [n + 400 for n in new], H, Hk, d, 16, seed=H + d)
    s.many = True
    _fill(d, 0.0)
    quiet = s.run(cap=CAP)
    for loud in (1e4, float("nan"), -3e4):
        _fill(d, loud)
        assert torch.equal(quiet, s.run(cap=CAP)), f"after queries of {loud}"


@pytest.mark.parametrize("H,Hk,d", [(8, 1, 128), (14, 2, 64), (4, 1, 256)])
def test_bits_do_not_depend_on_the_next_request(cuda_device, H, Hk, d):
    """A row tile holds the queries that come behind a request's last."""
    s = Paged([11, 60], [500, 200], H, Hk, d, 16, seed=H)
    s.many = True
    quiet = s.run(cap=CAP)[:11]
    s.q[11:] *= 4096.0
    assert torch.equal(quiet, s.run(cap=CAP)[:11])
    s.q[11:] = np.nan
    assert torch.equal(quiet, s.run(cap=CAP)[:11])
