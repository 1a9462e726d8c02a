"""emb_paged_slots against the token-by-token oracle: whole numbers, equal in every place."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_02501_gb300 as emb

pytestmark = pytest.mark.gpu


def _case(cached, added, page, max_pages, n_tokens=None, free=None, used=0, seed=0, holes=False):
    rng = np.random.default_rng(seed)
    R = len(cached)
    have = [min(-(-max(0, c) // page), max_pages) for c in cached]
    need = sum(min(-(-(max(0, c) + max(0, a)) // page), max_pages) - h for c, a, h in zip(cached, added, have))
    perm = rng.permutation(sum(have) + need + used + 5)
    table = np.full((R, max_pages), -7)
    at = 0
    for r, h in enumerate(have):
        table[r, :h] = perm[at:at + h]
        at += h
    if holes:
        table[rng.random(table.shape) < 0.3] = -1
    free_pages = perm[at:] if free is None else perm[at:at + free]
    T = sum(max(0, a) for a in added) if n_tokens is None else n_tokens
    return cached, added, free_pages, used, page, table, T


def _run(cached, added, free_pages, used, page, table, T, twice=True):
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()
    tab, R = i32(table), len(cached)
    q_start, kv = torch.full((R + 1,), -9, dtype=torch.int32, device="cuda"), torch.full((R,), -9, dtype=torch.int32, device="cuda")
    slots, pos = torch.full((T,), -9, dtype=torch.int64, device="cuda"), torch.full((T,), -9, dtype=torch.int32, device="cuda")
    used_out = torch.full((1,), -9, dtype=torch.int32, device="cuda")
    args = (i32(cached), i32(added), i32(free_pages), i32([used]), tab, q_start, kv, slots, pos, used_out, page)
    want = oracle.paged_slots_reference(cached, added, free_pages, used, page, table, T)
    for _ in range(2 if twice else 1):  # a repeated call changes nothing
        emb.emb_paged_slots(*args)
        torch.cuda.synchronize()
        for name, got, ref in zip(("table", "q_start", "kv_len", "slots", "positions"), (tab, q_start, kv, slots, pos), want):
            assert np.array_equal(got.cpu().numpy().astype(np.int64), ref), name
        assert int(used_out) == want[5]


@pytest.mark.parametrize("R,c_hi,a_hi,page", [(1, 0, 1, 16), (1, 816, 50, 16), (3, 40, 1, 16), (7, 100, 300, 32),
                                              (64, 2000, 2, 64), (255, 9, 9, 1), (257, 30, 20, 7), (1000, 500, 1, 16),
                                              (2000, 70, 3, 128), (5, 3000, 4000, 256), (300, 5, 700, 16)])
def test_random_lengths(cuda_device, R, c_hi, a_hi, page):
    rng = np.random.default_rng(R + page)
    cached, added = rng.integers(0, c_hi + 1, R).tolist(), rng.integers(0, a_hi + 1, R).tolist()
    if R == 1:
        cached, added = [c_hi], [a_hi]
    width = max(-(-(c + a) // page) for c, a in zip(cached, added)) + 2
    _run(*_case(cached, added, page, width, used=R % 5, seed=R))


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2049, 5000])
def test_one_request_over_several_blocks_of_tokens(cuda_device, n):
    _run(*_case([13], [n], 16, -(-(13 + n) // 16)))


def test_idle_and_negative_lengths(cuda_device):
    _run(*_case([0, 5, -3, 16, 0, 17], [0, 0, 4, -2, 33, 1], 16, 4))
    _run(*_case([0, 0], [0, 0], 16, 1))


@pytest.mark.parametrize("n_tokens", [0, 1, 30, 60, 200, 3000])
def test_padding_and_tokens_that_do_not_fit(cuda_device, n_tokens):
    """More token places than tokens (padding), and fewer (no slot, no page)."""
    _run(*_case([3, 0, 40], [20, 15, 30], 8, 20, n_tokens=n_tokens))


@pytest.mark.parametrize("free", [0, 1, 3])
def test_the_free_list_runs_out(cuda_device, free):
    _run(*_case([3, 0, 40], [20, 15, 30], 8, 20, free=free))


def test_requests_longer_than_their_row_of_the_table(cuda_device):
    _run(*_case([60, 0, 200], [20, 70, 3], 8, 8))


def test_entries_that_are_not_pages_give_no_slot(cuda_device):
    _run(*_case([30, 17, 90], [3, 20, 7], 8, 15, holes=True))


def test_unaligned_outputs(cuda_device):
    """slots and positions that start in the middle of a 16-byte line."""
    cached, added, free, used, page, table, T = _case([5, 9], [33, 40], 16, 6)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()
    slots = torch.zeros(T + 1, dtype=torch.int64, device="cuda")[1:]
    pos = torch.zeros(T + 3, dtype=torch.int32, device="cuda")[3:]
    out = [torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")]
    emb.emb_paged_slots(i32(cached), i32(added), i32(free), i32([used]), i32(table), *out, slots, pos,
                        torch.zeros(1, dtype=torch.int32, device="cuda"), page)
    want = oracle.paged_slots_reference(cached, added, free, used, page, table, T)
    assert np.array_equal(slots.cpu().numpy(), want[3]) and np.array_equal(pos.cpu().numpy(), want[4])
