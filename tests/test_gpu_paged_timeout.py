"""A join whose other part never comes: the wait gives up, the status says so once, and a workspace whose first 4 KB are
zeroed serves again."""
import pytest
import torch

import paper_2607_02501_gb300 as emb
from tests.paged_util import Paged

pytestmark = pytest.mark.gpu


def test_join_that_gives_up(cuda_device):
    s = Paged([1, 300], [20000, 900], 8, 1, 128, 64, seed=1)  # (with joins)
    want = s.run()
    ws = emb.paged_workspace()
    assert emb.emb_paged_status() == emb.EMB_OK
    emb.emb_paged_selftest_wait_timeout(ws, 2_000_000)  # 2 ms
    assert emb.emb_paged_status() == emb.EMB_ETIMEOUT
    assert emb.emb_paged_status() == emb.EMB_OK  # cleared
    assert int(ws[:4096].view(torch.int32).abs().sum()) != 0  # the part that was published
    ws[:4096].zero_()
    assert torch.equal(s.run(workspace=ws), want)
