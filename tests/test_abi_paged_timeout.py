"""What emb_paged_selftest_wait_timeout refuses (CPU only)."""
import pytest

import paper_2607_02501_gb300 as emb

WS = 0x7f0000000000


@pytest.mark.parametrize("ws,size,ns,want", [
    (None, emb.EMB_PAGED_WORKSPACE, 2000, "EINVAL"), (WS, emb.EMB_PAGED_WORKSPACE, 999, "EINVAL"), (WS, emb.EMB_PAGED_WORKSPACE, 10 ** 9 + 1, "EINVAL"),
    (WS + 128, emb.EMB_PAGED_WORKSPACE, 2000, "EALIGN"), (WS, emb.EMB_PAGED_WORKSPACE - 1, 2000, "ENOSPC")])
def test_refusals(ws, size, ns, want):
    emb.build()
    assert emb.paged_lib().emb_paged_selftest_wait_timeout(ws, size, ns, None) == getattr(emb, "EMB_" + want)
