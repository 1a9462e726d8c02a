"""Starts that no step has: whatever q_start holds, a call ends, reports nothing, and the next one is right."""
import numpy as np
import pytest
import torch

import paper_2607_02501_gb300 as emb
from tests.paged_util import Paged, dev_i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_q", [1, 4096])  # the kernel for few rows, and for many
@pytest.mark.parametrize("d", [64, 256])
def test_requests_that_claim_the_same_tokens(cuda_device, max_q, d):
    """Twenty thousand requests of all 4096 tokens each: their units of work pass 32 bits."""
    T, R, H = 4096, 40000, 8
    rng = np.random.default_rng(d)
    q = torch.randn(T, H * d, device="cuda").to(torch.bfloat16)
    cache = torch.randn(8, 64, H, d, device="cuda").to(torch.bfloat16)
    table = dev_i32(np.tile(rng.integers(0, 8, 64), (R, 1)))
    ws, O = emb.paged_workspace(), torch.empty_like(q)
    for starts in (np.arange(R + 1) % 2 * T, rng.integers(-5, T + 5, R + 1), rng.integers(-(2 ** 31), 2 ** 31 - 1, R + 1)):
        emb.emb_paged_attention(q, cache, cache, table, dev_i32(starts), dev_i32(np.full(R, 4096)), O, 0.1, max_q, ws)
        torch.cuda.synchronize()
        assert emb.emb_paged_status() == emb.EMB_OK
        assert int(ws[:4096].view(torch.int32).abs().sum()) == 0
    s = Paged([70, 1, 300], [90, 4000, 400], 8, 2, d, 16, seed=1)
    assert torch.equal(s.run(workspace=ws), s.run())
