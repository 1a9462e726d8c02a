"""emb_paged8_attention without padding: hints that take one call to either kernel, and lengths and starts beyond the buffers in the
kernel for many rows."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_02501_gb300 as emb
from tests.paged_util import host
from tests.paged8_util import F16_WEIGHT, Paged8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("mask", [{}, {"window": 90}, {"cap": 30.0}])
def test_the_hint_picks_the_kernel_only(cuda_device, mask, d):
    """1 and 2: up to 16 rows, the kernel for few; 200 and more: 1600 rows over too many tiles for clusters, the kernel for many."""
    s = Paged8([200, 3], [6200, 40], 8, 1, d, 64, seed=d)
    s.garble_unused()
    ws = emb.paged_workspace()
    outs = [s.check(F16_WEIGHT, max_q=hint, pad=pad, workspace=ws, **mask) for hint in (1, 2, 200, 10 ** 6) for pad in (0, 70)]
    for a, b in zip(outs[::2], outs[1::2]):
        assert torch.equal(a, b[:a.shape[0]])
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[4], outs[6])
    assert not torch.equal(outs[0], outs[4])  # (another kernel, other roundings)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_lengths_and_starts_beyond_the_buffers(cuda_device, d):
    s = Paged8([200, 90], [4000, 4000], 4, 1, d, 16, seed=24)
    sane = s.check(F16_WEIGHT, max_q=290)
    s.kv, s.q_start = [4000, 4000 + 500], np.array([0, 200, 290 + 900])
    assert torch.equal(s.run(max_q=290), sane)
    s.kv, s.q_start = [2 ** 31 - 1, 4000], np.array([-7, 200, 2 ** 31 - 1])
    assert torch.equal(s.run(max_q=10 ** 6), sane)
    # starts that go back: no queries; rows that the padding claims too are left out
    s.kv, s.q_start = [4000, 4000], np.array([0, 200, 120])
    ref, bound = oracle.paged_attention_reference(s.q, s.k, s.v, s.table, [0, 200, 200], s.kv, 4, s.scale, weight_error=F16_WEIGHT)
    assert (np.abs(host(s.run(max_q=200)) - ref) <= bound)[:120].all()
