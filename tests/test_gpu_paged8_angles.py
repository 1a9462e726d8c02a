"""The store's cosines and sines are within 1e-6, seen where the two products of a turned element cancel: what is left of it then is
their error, which bf16 keeps."""
import math

import numpy as np
import pytest
import torch

import paper_2607_02501_gb300 as emb
from tests.paged_util import dev_bf16, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("rot_dim", [64, 56])  # sixteen and eight elements a thread
@pytest.mark.parametrize("position", [1, -1, 12345, 2 ** 31 - 1, 1 - 2 ** 31])
@pytest.mark.parametrize("factor", [1.0, 0.5, 3.0])
def test_cosines_and_sines(cuda_device, factor, position, rot_dim, neighbours):
    """Bound: 1e-6 of both products, a rounding for the factor and one a product, and the output's to bf16."""
    d, half, T = 64, rot_dim // 2, 40
    rng = np.random.default_rng(rot_dim + position % 1000)
    a = rng.integers(128, 256, half) / 128.0 * rng.choice([-1, 1], half)  # (bf16)
    b = rng.integers(128, 256, half) / 128.0 * rng.choice([-1, 1], half)
    first = np.arange(half) * (2 if neighbours else 1)
    second = first + (1 if neighbours else half)
    inverse = pow(position % 2 ** 64, -1, 2 ** 64)
    worst = 0.0
    for which in range(2):
        # the angle at which the first, or the second, element vanishes, and the turns that give it at this position
        theta = [math.atan2(x, y) if which == 0 else math.atan2(-y, x) for x, y in zip(a, b)]
        units = [int(t / (2 * math.pi) * 2 ** 64) % 2 ** 64 for t in theta]
        turns = [u * inverse % 2 ** 64 for u in units]
        signed = torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turns], dtype=torch.int64).cuda()
        x = np.zeros((T, d))
        x[:, first], x[:, second] = a, b
        q, out = dev_bf16(x), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
        cache = emb.paged8_cache(3, 16, 1, d)
        emb.emb_paged8_store(q, q, q, out, *cache, torch.arange(T, device="cuda"), torch.full((T,), position, dtype=torch.int32, device="cuda"),
                             signed, neighbours=neighbours, factor=factor)
        turned = 2 * np.pi * np.array([(u - 2 ** 64 if u >= 2 ** 63 else u) / 2 ** 64 for u in units])
        want = factor * (a * np.cos(turned) - b * np.sin(turned) if which == 0 else b * np.cos(turned) + a * np.sin(turned))
        assert (np.abs(want) < 1e-14).all()
        got = host(out)[:, first if which == 0 else second]
        bound = factor * (np.abs(a) + np.abs(b)) * (1e-6 + 2 * 2.0 ** -24) * (1 + 2.0 ** -8)
        worst = max(worst, (np.abs(got - want) / (factor * (np.abs(a) + np.abs(b)))).max())
        assert (np.abs(got - want) <= bound).all(), worst
        assert (np.abs(got) > 0).any()  # (an error is seen at all)
