"""emb_paged8_attention against the oracle over the codes' values: the bf16 cache's cases of heads, pages, requests and masks, blocks
whose powers of two differ widely, NaN codes in hidden and visible places, exponent bytes of any value, queries of any
magnitude, padding, recorded calls, other streams, caches beyond 2^32 bytes."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_02501_gb300 as emb
from tests.paged_util import dev_bf16, dev_i32, host
from tests.paged8_util import F16_WEIGHT, Paged8, dev_u8
from tests.test_gpu_paged_attention import CASES

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["small", "many"], autouse=True)
def kernel(request):
    """Every test by the kernel that its sizes take, and by the one for many rows."""
    Paged8.many = request.param == "many"
    yield request.param
    Paged8.many = False


@pytest.mark.parametrize("new,kv,H,Hk,d,page", CASES)
@pytest.mark.parametrize("mask", ["causal", "prefix", "window", "capped", "wide cap"])
def test_parity(cuda_device, new, kv, H, Hk, d, page, mask):
    s = Paged8(new, kv, H, Hk, d, page, seed=len(new) + sum(kv) + d)
    s.garble_unused()
    prefix = [(2 * n) // 3 for n in kv] if mask == "prefix" else None
    kw = {"window": 70} if mask == "window" else {"cap": 30.0} if mask == "capped" else {"cap": 100.0} if mask == "wide cap" else {}
    s.check(F16_WEIGHT, prefix=prefix, what=f"{mask} new={new} kv={kv} H={H} Hk={Hk} d={d} page={page}", **kw)


@pytest.mark.parametrize("R", [64, 65, 400])
@pytest.mark.parametrize("q_hi", [1, 3, 40])
def test_many_requests(cuda_device, R, q_hi):
    """More requests than a warp shares out by itself, some idle, some without keys."""
    rng = np.random.default_rng(R + q_hi)
    new = rng.integers(0, q_hi + 1, R)
    kv = new + rng.integers(0, 90, R) * (rng.random(R) < 0.8)
    new[0] = kv[0] = q_hi
    s = Paged8(new.tolist(), kv.tolist(), 8, 2, 64, 16, seed=R)
    s.garble_unused()
    s.check(F16_WEIGHT, pad=5)


@pytest.mark.parametrize("d,H,new,kv", [(128, 8, 1, 20000), (64, 4, 2, 50000), (256, 2, 1, 9000), (128, 4, 20, 20000), (256, 8, 30, 6000)])
def test_long_histories(cuda_device, d, H, new, kv):
    """One item shared by as many CTAs as may join one."""
    s = Paged8([new], [kv], H, 1, d, 64, seed=kv)
    s.check(F16_WEIGHT)
    s.check(F16_WEIGHT, window=kv // 2, cap=30.0)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 150])
@pytest.mark.parametrize("spread", [3, 30])
def test_blocks_of_unlike_powers(cuda_device, d, new, spread):
    """Values between 2^-30 and 2^30 by block: a query's output is that of the few blocks with the largest, and within them exact.
    (Keys spread by 2^3 at most: scores beyond that leave one key.)"""
    s = Paged8([new, new], [new + 333, new], 4, 2, d, 32, seed=19, spread=spread)
    s.k = np.clip(s.k, -8, 8)
    s.check(F16_WEIGHT)
    s.check(F16_WEIGHT, window=50, cap=20.0)
    # a dominant key whose values are the smallest: the scores' sum counts it in full
    s = Paged8([new], [new + 200], 4, 2, d, 32, seed=20)
    s.q = np.abs(s.q)
    pos = 100
    pg, at = s.at(0, pos)
    s.k[pg, at] = 4.0
    s.v[pg, at // 16 * 16:at // 16 * 16 + 16] *= 2.0 ** -40
    s.check(F16_WEIGHT)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 150])
def test_exponent_bytes_of_any_value(cuda_device, d, new):
    """Bytes beyond the range count as its ends."""
    outs = []
    for far, near in ((0, 79), (255, 175)):
        for byte in (far, near):
            s = Paged8([new], [new + 100], 4, 2, d, 16, seed=21)
            s.encode()
            s.codes[3][:, :, 0] = byte  # values of one head
            s.codes[2][:, :, 1] = 79 if byte in (0, 79) else 127
            s.codes[2][0, 0, 1] = 0 if byte == 0 else s.codes[2][0, 0, 1]
            s.settle()
            outs.append(host(s.check(F16_WEIGHT)))
        assert np.array_equal(outs[-1], outs[-2])


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 150])
def test_queries_of_any_magnitude(cuda_device, d, new):
    """Rows of one call from 2^-60 to 2^60, scaled so that the scores are ordinary for some of them; rows of zeros."""
    s = Paged8([new], [new + 100], 4, 2, d, 16, seed=22)
    by = 2.0 ** s.rng.integers(-60, 61, (s.q.shape[0], 4, 1))
    by[0, 0] = 0.0
    s.q = (s.q.reshape(-1, 4, d) * by).reshape(s.q.shape)
    s.check(F16_WEIGHT)
    s.scale *= 2.0 ** -55
    s.check(F16_WEIGHT)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 500])
@pytest.mark.parametrize("new", [1, 5, 150])
def test_windows(cuda_device, d, window, new):
    s = Paged8([new, new], [new + 400, new], 4, 2, d, 16, seed=window)
    s.garble_unused()
    s.check(F16_WEIGHT, window=window, cap=20.0 if window == 16 else 0.0)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 6], [6, 3], [100, 40]])
def test_full_and_beyond(cuda_device, d, new):
    """A prefix as long as the request hides nothing; longer or negative ones count as that or none."""
    kv = [n + 77 for n in new]
    s = Paged8(new, kv, 4, 2, d, 16, seed=5)
    full = s.check(F16_WEIGHT, prefix=kv)
    assert torch.equal(full, s.run(prefix=[n + 1000 for n in kv]))
    assert torch.equal(s.run(prefix=[-4, -1]), s.run())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,kv", [([4], [0]), ([5, 3], [2, 0]), ([40, 2], [3, 9]), ([200], [50]), ([1], [0])])
def test_queries_without_a_key_give_zeros(cuda_device, d, new, kv):
    s = Paged8(new, kv, 4, 2, d, 16, seed=6)
    s.garble_unused()
    O = s.check(F16_WEIGHT, pad=3)
    assert (host(O)[:max(0, new[0] - kv[0])] == 0).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,kv", [([6], [40]), ([3], [130]), ([150], [150]), ([70], [300])])
@pytest.mark.parametrize("bad", [0x7F, 0xFF])
def test_nan_codes(cuda_device, d, new, kv, bad):
    """A NaN code has no part in the queries that do not see it: its row is visible from its own position on (causal), so earlier
    queries stay as they are."""
    s = Paged8(new, kv, 4, 2, d, 16, seed=8)
    clean = host(s.run())
    pos = kv[0] - new[0] // 2 - 1
    first = pos - (kv[0] - new[0])  # the query at the spoilt token
    pg, at = s.at(0, pos)
    kc, vc = s.codes[0], s.codes[1]
    v0, k0 = vc[pg, at].copy(), kc[pg, at].copy()
    vc[pg, at, 1, 3] = bad
    O = host(s.run())
    assert np.array_equal(O[:first], clean[:first])
    cols = np.zeros(4 * d, dtype=bool)
    cols[[2 * d + 3, 3 * d + 3]] = True
    assert np.isnan(O[first:][:, cols]).all()
    assert np.array_equal(O[:, ~cols], clean[:, ~cols])
    vc[pg, at] = v0
    kc[pg, at, 0] = bad
    O = host(s.run())
    assert np.array_equal(O[:first], clean[:first])
    assert np.isnan(O[first:, :2 * d]).all() and np.array_equal(O[:, 2 * d:], clean[:, 2 * d:])
    # behind a window it is hidden from later queries too
    kc[pg, at], vc[pg, at] = bad, bad
    O = host(s.run(window=2))
    rest = np.ones(new[0], dtype=bool)
    rest[first:first + 2] = False
    vc[pg, at], kc[pg, at] = v0, k0
    assert np.array_equal(O[rest], host(s.run(window=2))[rest]) and np.isnan(O[~rest]).all()


@pytest.mark.parametrize("new", [1, 6, 120])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_queries_that_are_not_finite(cuda_device, new, bad):
    """One element of one query's head: that row of the output is NaN (an infinite one gives scores of both signs), others stay."""
    s = Paged8([new], [new + 200], 2, 1, 128, 16, seed=9)
    clean = host(s.run())
    s.q[0, 5] = bad
    O = host(s.run())
    assert np.isnan(O[0, :128]).all()
    O[0, :128] = clean[0, :128]
    assert np.array_equal(O, clean)


def test_pages_that_do_not_exist_count_as_zeros(cuda_device):
    for new in (1, 5, 100):
        s = Paged8([new], [new + 300], 4, 1, 128, 16, seed=10)
        s.encode()
        s.table[0, 3], s.table[0, 7] = -1, s.k.shape[0] + 5
        s.check(F16_WEIGHT)


@pytest.mark.parametrize("new,kv,H,Hk,d", [([1, 1], [2000, 31], 8, 1, 128), ([9, 1], [700, 50], 8, 2, 64), ([200, 3], [900, 3], 8, 2, 128),
                                           ([80], [400], 8, 1, 256)])
def test_reproducible_padded_and_any_hint(cuda_device, new, kv, H, Hk, d):
    s = Paged8(new, kv, H, Hk, d, 32, seed=11)
    ws = emb.paged_workspace()
    O = s.check(F16_WEIGHT, pad=70, workspace=ws)
    for _ in range(3):
        assert torch.equal(O, s.run(pad=70, workspace=ws))
    for hint in (1, 4, 10 ** 6):  # the hint picks the kernel only
        s.check(F16_WEIGHT, max_q=hint, workspace=ws)


def test_lengths_and_starts_beyond_the_buffers(cuda_device):
    s = Paged8([2, 3], [64, 64], 4, 2, 128, 16, seed=12)
    s.many = False  # (no padding: the starts are to pass the tokens)
    s.kv = [64, 64 + 500]
    s.q_start = np.array([0, 2, 5 + 90])
    a = host(s.run())
    s.kv, s.q_start = [64, 64], np.array([0, 2, 5])
    assert np.array_equal(a, host(s.run()))
    s.q_start = np.array([0, 5, 2])  # decreasing: no queries, rows of no request are the padding
    ref, bound = oracle.paged_attention_reference(s.q, s.k, s.v, s.table, [0, 5, 5], s.kv, 4, s.scale, weight_error=F16_WEIGHT)
    out = host(s.run(max_q=5))
    assert (np.abs(out - ref) <= bound)[:2].all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 9, 130])
@pytest.mark.parametrize("scale,cap", [(-0.1, 0.0), (-0.1, 3.0), (0.0, 0.0), (0.0, 5.0), (0.5, 1.0)])
def test_scales_of_any_sign_and_tight_caps(cuda_device, d, new, scale, cap):
    s = Paged8([new], [new + 150], 4, 2, d, 16, seed=18)
    s.garble_unused()
    s.scale = scale
    s.check(F16_WEIGHT, cap=cap, window=40)


def test_strong_scores_and_large_gains(cuda_device):
    for new in (1, 4, 90):
        s = Paged8([new], [new + 500], 4, 1, 128, 16, seed=13, gain=30.0)
        s.check(F16_WEIGHT)
        s.check(F16_WEIGHT, cap=50.0)


def test_growing_scores(cuda_device):
    """Each tile's scores exceed the last's, so the running maximum moves in every tile."""
    for new in (1, 8, 140):
        s = Paged8([new], [1200], 2, 1, 128, 16, seed=14)
        for pos in range(1200):
            pg, at = s.at(0, pos)
            s.k[pg, at] = s.k[pg, at] * 0.01 + pos / 100.0
        s.q = np.abs(s.q) * 0.25
        s.check(F16_WEIGHT, prefix=[1200])


@pytest.mark.parametrize("new", [1, 20, 130])
def test_recorded_call_follows_its_lengths(cuda_device, new):
    """A recorded call reads lengths, table, codes and exponents at every replay; an eager one goes on beside it."""
    s = Paged8([new, new], [new + 600, new + 40], 4, 2, 128, 16, seed=15)
    s.encode()
    pad = 6000 if Paged8.many else 0
    q, hint = dev_bf16(np.concatenate([s.q, np.zeros((pad, s.q.shape[1]), dtype=np.float32)])), pad or new
    cache, tab, qs, kv = [dev_u8(c) for c in s.codes], dev_i32(s.table), dev_i32(s.q_start), dev_i32(s.kv)
    O, ws, stream = torch.empty_like(q), emb.paged_workspace(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with emb.Recording(stream, keep=[q, cache, tab, qs, kv, O, ws]) as rec:
        emb.emb_paged8_attention(q, *cache, tab, qs, kv, O, s.scale, hint, ws, stream=stream)
    for lens in ([new + 600, new + 40], [new, new + 39], [new + 300, new]):
        s.kv = lens
        s.codes[3] += 1
        with torch.cuda.stream(stream):
            kv.copy_(dev_i32(lens))
            cache[3].copy_(dev_u8(s.codes[3]))
            rec.launch(stream)
        torch.cuda.synchronize()
        assert torch.equal(O[:s.T], s.run())
    rec.close()


def test_on_another_stream_than_the_current(cuda_device):
    s = Paged8([1, 70], [500, 300], 8, 2, 128, 16, seed=16)
    assert torch.equal(s.run(), s.run(stream=torch.cuda.Stream()))


@pytest.mark.parametrize("new", [1, 100])
def test_cache_beyond_32_bits(cuda_device, new):
    """Pages whose byte offsets pass 2^32, in all three operators."""
    Hk, d, page = 8, 128, 64
    n_pages = (1 << 33) // (page * Hk * d)
    s = Paged8([new], [new + 200], Hk, Hk, d, page, seed=17)
    codes = s.encode()
    n = s.table.shape[1]
    cache = emb.paged8_cache(n_pages, page, Hk, d)
    far = np.array([[n_pages - 1 - 3 * i for i in range(n)]])
    for i in range(n):
        for to, x in zip(cache, codes):
            to[far[0, i]] = dev_u8(x[s.table[0, i]])
    pad = 6000 if Paged8.many else 0
    q, hint = dev_bf16(np.concatenate([s.q, np.zeros((pad, s.q.shape[1]), dtype=np.float32)])), pad or new
    O = torch.empty_like(q)
    emb.emb_paged8_attention(q, *cache, dev_i32(far), dev_i32(s.q_start), dev_i32(s.kv), O, s.scale, hint, emb.paged_workspace())
    assert torch.equal(O[:s.T], s.run())
    slots = torch.tensor([(n_pages - 1) * page + 16], dtype=torch.int64, device="cuda")
    x = torch.randn(1, Hk * d, device="cuda").to(torch.bfloat16)
    emb.emb_paged8_store(x, x, x, torch.empty_like(x), *cache, slots, torch.zeros(1, dtype=torch.int32, device="cuda"), None)
    ko, vo = torch.empty_like(x), torch.empty_like(x)
    emb.emb_paged8_read(*cache, slots, ko, vo)
    assert torch.equal(ko, vo) and ((ko.float() - x.float()).abs() <= 2.0 ** -4 * x.float().abs() + 1e-3).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 150])
def test_scores_near_the_largest_numbers(cuda_device, d, new):
    """Scores of up to 2^125 whose order hangs on the blocks' powers: one key has all the weight."""
    s = Paged8([new], [new + 60], 2, 1, d, 16, seed=23)
    s.q = np.full_like(s.q, 2.0 ** 97)
    s.k = np.zeros_like(s.k)
    far, near = s.at(0, 5), s.at(0, 40)
    s.k[far][0, 0] = 2.0 ** 28          # by a large block's smallest code: 2^125
    s.k[far[0], (far[1] + 1) % 16, 0, 1] = 2.0 ** 34
    s.k[near][0, :4] = 2.0 ** 24        # by a small block's largest: 2^123
    s.scale = 1.0
    s.q[:, 1::d] = 0.0                  # (the element that makes the first block large does not count)
    O = host(s.run())
    assert np.array_equal(O, np.tile(oracle.paged8_values(s.codes[1], s.codes[3])[far][0], (new, 2)))
