"""emb_paged8_attention's kernel for many rows where one of an item's two row tiles has no query, or sees few of the tiles that the
other one walks: its warps pass over tiles while the others work, however far ahead or behind, and come back in step."""
import pytest
import torch

import paper_2607_02501_gb300 as emb
from tests.paged8_util import F16_WEIGHT, Paged8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,kv,H,window", [
    ([16, 5, 1], [9000, 700, 4000], 8, 0),      # one row tile of 16 queries of 8 heads: the other has none
    ([40, 33], [6000, 2500], 8, 0),             # the last block has one row tile, or one query in the second
    ([300], [5000], 8, 20),                     # a window: each row tile sees a tile or two of its own
    ([64, 64], [3000, 40], 4, 600),             # the first tiles are the first row tile's alone, the last the second's
    ([20], [10], 16, 0)])                       # queries before the first key: a row tile without any key
def test_row_tiles_that_pass_over_tiles(cuda_device, d, new, kv, H, window):
    s = Paged8(new, kv, H, 1, d, 16, seed=sum(kv) + d, spread=2)
    s.many = True
    ws = emb.paged_workspace()
    O = s.check(F16_WEIGHT, window=window, workspace=ws)
    for _ in range(20):
        assert torch.equal(O, s.run(window=window, workspace=ws))
