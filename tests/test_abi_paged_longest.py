"""Block tables whose last keys' numbers would pass 31 bits once a tile is added are refused (CPU only: the calls fail their
validation)."""
import pytest

import paper_2607_02501_gb300 as emb
from tests.test_abi_paged import ATTN, _call


@pytest.mark.parametrize("max_pages,page", [((1 << 27) - 1, 16), ((1 << 27) - 31, 16), ((1 << 23) - 1, 256), (1 << 27, 16)])
def test_refused(max_pages, page):
    emb.build()
    assert _call(emb.paged_lib().emb_paged_attention, ATTN, {"max_pages": max_pages, "page": page, "n_req": 1, "T": 1}) == emb.EMB_EINVAL
