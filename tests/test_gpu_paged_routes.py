"""A cap does not change which kernel a call takes, nor how it shares out its work."""
import pytest
import torch

import paper_2607_02501_gb300 as emb
from tests.gpu_util import launches

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,H,Hk,d,new,keys,window", [
    (24, 14, 2, 64, 7, 3000, 1024), (40, 8, 4, 128, 1, 1200, 0), (30, 8, 4, 64, 1, 2100, 0), (20, 16, 2, 128, 3, 2500, 0), (60, 2, 2, 256, 1, 1300, 0),
    (1, 8, 1, 128, 1, 867, 0), (4, 32, 8, 128, 1, 9000, 0), (1, 8, 1, 128, 2000, 2000, 0), (12, 2, 2, 64, 7, 9800, 0), (64, 32, 8, 128, 1, 16000, 0)])
def test_same_route_with_and_without_a_cap(cuda_device, R, H, Hk, d, new, keys, window):
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.zeros(R * new, H * d, dtype=torch.bfloat16, device="cuda")
    cache = torch.zeros(2, 64, Hk, d, dtype=torch.bfloat16, device="cuda")
    args = (q, cache, cache, torch.zeros(R, -(-keys // 64), **i32), torch.arange(R + 1, **i32) * new, torch.full((R,), keys, **i32), torch.empty_like(q),
            0.1, new, emb.paged_workspace())
    got = []
    for cap in (0.0, 50.0, 500.0):
        emb.emb_paged_attention(*args, cap=cap, window=window)
        (name, template, grid), = launches(lambda: emb.emb_paged_attention(*args, cap=cap, window=window))
        got.append((name, template[0], template[2:], grid))  # all but the form of the scores
    assert got[0] == got[1] == got[2]
