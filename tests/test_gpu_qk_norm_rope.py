"""emb_qk_norm_rope against the oracle: head sizes, partial rotation, several position axes, with and
without norms, packed and separate projections, slots that store nothing; values are copied bit for bit
and nothing else of the cache changes."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_02501_gb300 as emb
from tests.paged_util import bf16, check, dev_bf16, host

pytestmark = pytest.mark.gpu
BASE, EPS = 10000.0, 1e-6


def _run(T, H, Hk, d, rot=None, axes=1, norm="qk", packed=False, page=16, seed=0, pos0=0, base=BASE, gain=1.0, drop=()):
    rng = np.random.default_rng(seed)
    rot = d if rot is None else rot
    x = [bf16(rng.standard_normal((T, h * d)) * gain) for h in (H, Hk, Hk)]
    if packed:
        m = dev_bf16(np.concatenate(x, axis=1))
        dev = m.split([H * d, Hk * d, Hk * d], dim=1)
    else:
        dev = [dev_bf16(a) for a in x]
    gammas = [(1 + 0.2 * rng.standard_normal(d)).astype(np.float32) if c in norm else None for c in "qk"]
    positions = pos0 + rng.integers(0, 900, (axes, T))
    positions[:, 0] = pos0
    axis = rng.integers(0, axes, rot // 2)
    n_pages = -(-T // page) + 2
    order = rng.permutation(n_pages)
    slots = order[np.arange(T) // page] * page + np.arange(T) % page
    for i, t in enumerate(drop):
        slots[t] = [-1, n_pages * page, -5, 1 << 40][i % 4]
    kc, vc = (bf16(rng.standard_normal((n_pages, page, Hk, d))) for _ in range(2))
    kd, vd = dev_bf16(kc), dev_bf16(vc)
    out = torch.full((T, H * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    emb.emb_qk_norm_rope(*dev, out, kd, vd, torch.from_numpy(slots.astype(np.int64)).cuda(),
                         torch.from_numpy(positions.astype(np.int32)).cuda(),
                         *[None if g is None else torch.from_numpy(g).cuda() for g in gammas], eps=EPS,
                         axis_of_pair=axis.tolist() if axes > 1 else None, rot_dim=rot, base=base)
    torch.cuda.synchronize()
    what = f"T={T} H={H} Hk={Hk} d={d} rot={rot} axes={axes} norm={norm}"
    check(host(out), *oracle.qk_norm_rope_reference(x[0], H, d, gammas[0], EPS, positions, axis, rot, base), "q " + what)
    ref, bound = oracle.qk_norm_rope_reference(x[1], Hk, d, gammas[1], EPS, positions, axis, rot, base)
    kh, vh = host(kd).reshape(-1, Hk * d), host(vd).reshape(-1, Hk * d)
    stored = (slots >= 0) & (slots < n_pages * page)
    check(kh[slots[stored]], ref[stored], bound[stored], "k " + what)
    kc, vc = kc.reshape(-1, Hk * d).copy(), vc.reshape(-1, Hk * d).copy()
    vc[slots[stored]] = x[2][stored]
    assert np.array_equal(vh, vc), "values, and the rest of the value cache"
    rest = np.ones(len(kc), dtype=bool)
    rest[slots[stored]] = False
    assert np.array_equal(kh[rest], kc[rest]), "the rest of the key cache"


@pytest.mark.parametrize("T,H,Hk,d", [(1, 8, 1, 128), (3, 1, 1, 8), (50, 8, 1, 256), (7, 14, 2, 64), (300, 32, 8, 128),
                                      (33, 16, 16, 72), (2, 5, 5, 200), (1000, 4, 4, 128), (17, 3, 1, 24)])
def test_sizes(cuda_device, T, H, Hk, d):
    _run(T, H, Hk, d, seed=T)


@pytest.mark.parametrize("norm", ["", "q", "k", "qk"])
@pytest.mark.parametrize("packed", [False, True])
def test_norms_and_packed_projections(cuda_device, norm, packed):
    _run(45, 8, 2, 128, norm=norm, packed=packed, seed=3)


@pytest.mark.parametrize("d,rot", [(128, 64), (64, 8), (256, 0), (80, 40), (128, 120), (72, 56)])
def test_partial_rotation(cuda_device, d, rot):
    _run(21, 4, 2, d, rot=rot, seed=rot)


@pytest.mark.parametrize("axes", [2, 3, 4])
def test_position_axes(cuda_device, axes):
    _run(40, 8, 2, 128, axes=axes, packed=True, seed=axes)


@pytest.mark.parametrize("pos0", [0, 4000, 1 << 20, (1 << 24) - 1000, (1 << 31) - 1000, -(1 << 20), -5])
def test_positions(cuda_device, pos0):
    _run(12, 2, 1, 64, pos0=pos0, seed=7)


@pytest.mark.parametrize("base", [0.5, 1.0, 1e6])
def test_bases(cuda_device, base):
    _run(12, 2, 1, 64, pos0=100, base=base, seed=8)


def test_slots_that_store_nothing(cuda_device):
    _run(30, 4, 2, 128, drop=(0, 7, 8, 29), seed=9)


def test_large_and_tiny_rows(cuda_device):
    _run(9, 4, 2, 128, gain=1e4, seed=10)
    _run(9, 4, 2, 128, gain=1e-4, seed=11)


def test_same_result_in_any_batch(cuda_device):
    """A token's outputs do not depend on how many come with it (one or several rows per thread)."""
    rng = np.random.default_rng(1)
    T, H, Hk, d = 4000, 8, 2, 128
    q, k, v = (dev_bf16(rng.standard_normal((T, h * d))) for h in (H, Hk, Hk))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    slots = torch.arange(T, dtype=torch.int64, device="cuda")
    g = torch.rand(d, device="cuda") + 0.5
    kc, vc = (torch.zeros(T // 16, 16, Hk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    all_q, one_q = torch.empty_like(q), torch.empty_like(q)
    emb.emb_qk_norm_rope(q, k, v, all_q, kc, vc, slots, pos, g, g)
    k_all = kc.clone()
    kc.zero_()
    for t in (0, 1234, 3999):
        emb.emb_qk_norm_rope(q[t:t + 1], k[t:t + 1], v[t:t + 1], one_q[t:t + 1], kc, vc, slots[t:t + 1], pos[t:t + 1], g, g)
        assert torch.equal(one_q[t], all_q[t]) and torch.equal(kc.view(T, -1)[t], k_all.view(T, -1)[t])
