"""emb_paged_attention against the oracle: one token to some hundred per request, ragged requests, every head and
page size, masks that hide whole tiles or leave a row empty, capped scores, NaN and infinities in hidden
places, caches beyond 2^32 bytes, padding, recorded calls and other streams."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_02501_gb300 as emb
from tests.paged_util import Paged, dev_bf16, dev_i32, host

pytestmark = pytest.mark.gpu
# rounding of the value product's weights: bf16 hi + lo, within the oracle's allowance, up to 16 rows of queries
# times heads per key/value head; one bf16 (2^-9, taken as 2^-8) above
ONE_BF16 = 2.0 ** -8


def _werr(new, H, Hk):
    return ONE_BF16 if Paged.many or max(new) * (H // Hk) > 16 else 0.0


@pytest.fixture(params=["small", "many"], autouse=True)
def kernel(request):
    """Every test by the kernel that its sizes take, and by the one for many rows."""
    Paged.many = request.param == "many"
    yield request.param
    Paged.many = False


CASES = [
    # new, kv, H, Hk, d, page
    ([1], [1], 1, 1, 64, 16),
    ([1], [867], 8, 1, 128, 16),
    ([1], [64], 8, 1, 256, 64),
    ([1, 1, 1], [5, 700, 64], 8, 2, 128, 32),
    ([1] * 40, list(range(1, 400, 10)), 4, 4, 64, 16),
    ([1, 0, 1, 0], [300, 17, 65, 0], 28, 4, 128, 16),
    ([1], [3000], 16, 1, 64, 128),
    ([1], [500], 32, 1, 128, 16),
    ([1, 1], [129, 1000], 64, 1, 64, 256),
    ([2, 5, 1], [100, 5, 333], 8, 1, 128, 16),
    ([7, 3], [7, 900], 14, 2, 64, 32),
    ([8], [1500], 8, 1, 256, 64),
    ([3, 4], [90, 400], 14, 2, 256, 16),
    ([50], [866], 8, 1, 128, 16),
    ([50, 20], [50, 300], 8, 1, 64, 16),
    ([130], [130], 4, 4, 128, 16),
    ([129, 1, 64, 0, 200], [129, 350, 500, 10, 777], 8, 2, 128, 64),
    ([300], [300], 7, 1, 64, 16),
    ([100, 33], [164, 33], 8, 1, 256, 16),
    ([257], [600], 2, 2, 256, 128),
    ([1, 90], [900, 90], 64, 1, 128, 32),
]


@pytest.mark.parametrize("new,kv,H,Hk,d,page", CASES)
@pytest.mark.parametrize("mask", ["causal", "prefix", "window", "capped"])
def test_parity(cuda_device, new, kv, H, Hk, d, page, mask):
    s = Paged(new, kv, H, Hk, d, page, seed=len(new) + sum(kv) + d)
    s.spoil_unused()
    prefix = [(2 * n) // 3 for n in kv] if mask == "prefix" else None
    kw = {"window": 70} if mask == "window" else {"cap": 30.0} if mask == "capped" else {}
    s.check(_werr(new, H, Hk), prefix=prefix, what=f"{mask} new={new} kv={kv} H={H} Hk={Hk} d={d} page={page}", **kw)


@pytest.mark.parametrize("R", [64, 65, 130, 400])
@pytest.mark.parametrize("q_hi", [1, 3, 40])
def test_many_requests(cuda_device, R, q_hi):
    """More requests than a warp shares out by itself, some idle, some without keys."""
    rng = np.random.default_rng(R + q_hi)
    new = rng.integers(0, q_hi + 1, R)
    kv = new + rng.integers(0, 90, R) * (rng.random(R) < 0.8)
    new[0] = kv[0] = q_hi
    s = Paged(new.tolist(), kv.tolist(), 8, 2, 64, 16, seed=R)
    s.spoil_unused()
    s.check(_werr([q_hi], 8, 2), pad=5)


@pytest.mark.parametrize("d,H,new,kv", [(128, 8, 1, 20000), (64, 4, 2, 50000), (256, 2, 1, 9000), (128, 4, 20, 20000), (256, 8, 30, 6000)])
def test_long_histories(cuda_device, d, H, new, kv):
    """One item shared by as many CTAs as may join one."""
    s = Paged([new], [kv], H, 1, d, 64, seed=kv)
    s.check(_werr([new], H, 1))
    s.check(_werr([new], H, 1), window=kv // 2, cap=30.0)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 500])
@pytest.mark.parametrize("new", [1, 5, 150])
def test_windows(cuda_device, d, window, new):
    s = Paged([new, new], [new + 400, new], 4, 2, d, 16, seed=window)
    s.spoil_unused()
    s.check(_werr([new], 4, 2), window=window, cap=20.0 if window == 16 else 0.0)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 6], [6, 3], [100, 40]])
def test_full_and_beyond(cuda_device, d, new):
    """A prefix as long as the request hides nothing; longer or negative ones count as that or none."""
    kv = [n + 77 for n in new]
    s = Paged(new, kv, 4, 2, d, 16, seed=5)
    full = s.check(_werr(new, 4, 2), prefix=kv)
    assert torch.equal(full, s.run(prefix=[n + 1000 for n in kv]))
    assert torch.equal(s.run(prefix=[-4, -1]), s.run())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,kv", [([4], [0]), ([5, 3], [2, 0]), ([40, 2], [3, 9]), ([200], [50]), ([1], [0])])
def test_queries_without_a_key_give_zeros(cuda_device, d, new, kv):
    """Fewer keys than queries: the first queries lie before position 0 and see nothing."""
    s = Paged(new, kv, 4, 2, d, 16, seed=6)
    s.spoil_unused()
    O = s.check(_werr(new, 4, 2), pad=3)
    assert (host(O)[:max(0, new[0] - kv[0])] == 0).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,kv", [([6], [40]), ([3], [130]), ([150], [150]), ([70], [300])])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_hidden_values_that_are_not_finite(cuda_device, d, new, kv, bad):
    """A key and a value that is not finite has no part in the queries that do not see it: its row is
    visible from its own position on (causal), so earlier queries stay as they are."""
    s = Paged(new, kv, 4, 2, d, 16, seed=8)
    clean = host(s.run())
    pos = kv[0] - new[0] // 2 - 1
    first = pos - (kv[0] - new[0])  # the query at the spoilt token
    pg, at = s.at(0, pos)
    v0, k0 = s.v[pg, at].copy(), s.k[pg, at].copy()
    s.v[pg, at, 1, 3] = bad
    O = host(s.run())
    assert np.array_equal(O[:first], clean[:first])
    cols = np.zeros(4 * d, dtype=bool)
    cols[[2 * d + 3, 3 * d + 3]] = True
    assert not np.isfinite(O[first:][:, cols]).any()
    assert np.array_equal(O[:, ~cols], clean[:, ~cols])
    s.v[pg, at] = v0
    s.k[pg, at, 0] = bad if np.isnan(bad) else np.nan
    O = host(s.run())
    assert np.array_equal(O[:first], clean[:first])
    assert np.isnan(O[first:, :2 * d]).all() and np.array_equal(O[:, 2 * d:], clean[:, 2 * d:])
    # behind a window it is hidden from later queries too
    s.k[pg, at] = k0
    s.v[pg, at] = np.nan
    s.k[pg, at] = np.nan
    O = host(s.run(window=2))
    rest = np.ones(new[0], dtype=bool)
    rest[first:first + 2] = False
    s.v[pg, at], s.k[pg, at] = v0, k0
    assert np.array_equal(O[rest], host(s.run(window=2))[rest]) and np.isnan(O[~rest]).all()


@pytest.mark.parametrize("new", [1, 6, 120])
def test_scores_that_are_not_finite(cuda_device, new):
    s = Paged([new], [new + 200], 2, 1, 128, 16, seed=9)
    s.q[:, :128] = np.abs(s.q[:, :128])
    # a key of -infinity everywhere: score -infinity for head 0 (weight zero), so as if the key were not there
    pg, at = s.at(0, 30)
    s.k[pg, at] = -np.inf
    with_key = host(s.run())[:, :128]
    s.k[pg, at] = 0
    assert np.isfinite(with_key).all()
    s.k[pg, at] = np.inf
    assert np.isnan(host(s.run())[:, :128]).all()


def test_pages_that_do_not_exist_count_as_zeros(cuda_device):
    for new in (1, 5, 100):
        s = Paged([new], [new + 300], 4, 1, 128, 16, seed=10)
        s.table[0, 3], s.table[0, 7] = -1, s.k.shape[0] + 5
        s.check(_werr([new], 4, 1))


@pytest.mark.parametrize("new,kv,H,Hk,d", [([1, 1], [2000, 31], 8, 1, 128), ([9, 1], [700, 50], 8, 2, 64), ([200, 3], [900, 3], 8, 2, 128),
                                           ([80], [400], 8, 1, 256)])
def test_reproducible_padded_and_any_hint(cuda_device, new, kv, H, Hk, d):
    s = Paged(new, kv, H, Hk, d, 32, seed=11)
    ws = emb.paged_workspace()
    O = s.check(_werr(new, H, Hk), pad=70, workspace=ws)
    for _ in range(3):
        assert torch.equal(O, s.run(pad=70, workspace=ws))
    for hint in (1, 4, 10 ** 6):  # the hint picks the kernel only
        s.check(ONE_BF16, max_q=hint, workspace=ws)


def test_lengths_and_starts_beyond_the_buffers(cuda_device):
    """kv_len past the table's row counts as the row's end, starts past n_tokens as n_tokens."""
    s = Paged([2, 3], [64, 64], 4, 2, 128, 16, seed=12)
    s.many = False  # (no padding: the starts are to pass the tokens)
    s.kv = [64, 64 + 500]
    s.q_start = np.array([0, 2, 5 + 90])
    a = host(s.run())
    s.kv, s.q_start = [64, 64], np.array([0, 2, 5])
    assert np.array_equal(a, host(s.run()))
    s.q_start = np.array([0, 5, 2])  # decreasing: no queries, rows of no request are the padding
    s.kv = [64, 64]
    ref, bound = oracle.paged_attention_reference(s.q, s.k, s.v, s.table, [0, 5, 5], s.kv, 4, s.scale)
    out = host(s.run(max_q=5))
    assert (np.abs(out - ref) <= bound)[:2].all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 9, 130])
@pytest.mark.parametrize("scale,cap", [(-0.1, 0.0), (-0.1, 3.0), (0.0, 0.0), (0.0, 5.0), (0.5, 1.0)])
def test_scales_of_any_sign_and_tight_caps(cuda_device, d, new, scale, cap):
    """A negative or zero scale; a cap so tight that a hidden key taken as -cap would show."""
    s = Paged([new], [new + 150], 4, 2, d, 16, seed=18)
    s.spoil_unused()
    s.scale = scale
    s.check(_werr([new], 4, 2), cap=cap, window=40)


def test_strong_scores_and_large_gains(cuda_device):
    for new in (1, 4, 90):
        s = Paged([new], [new + 500], 4, 1, 128, 16, seed=13, gain=30.0)
        s.check(_werr([new], 4, 1))
        s.check(_werr([new], 4, 1), cap=50.0)


def test_growing_scores(cuda_device):
    """Each tile's scores exceed the last's, so the running maximum moves in every tile."""
    for new in (1, 8, 140):
        s = Paged([new], [1200], 2, 1, 128, 16, seed=14)
        for pos in range(1200):
            pg, at = s.at(0, pos)
            s.k[pg, at] = s.k[pg, at] * 0.01 + pos / 100.0
        s.q = np.abs(s.q) * 0.25
        from tests.paged_util import bf16
        s.k, s.q = bf16(s.k), bf16(s.q)
        s.check(_werr([new], 2, 1), prefix=[1200])


def _rows_and_hint(s, new):
    """Queries on the device and the hint, padded as Paged.run pads them."""
    pad = 6000 if Paged.many else 0
    return dev_bf16(np.concatenate([s.q, np.zeros((pad, s.q.shape[1]), dtype=np.float32)])), pad or new


@pytest.mark.parametrize("new", [1, 20, 130])
def test_recorded_call_follows_its_lengths(cuda_device, new):
    """A recorded call reads lengths, table and queries at every replay."""
    s = Paged([new, new], [new + 600, new + 40], 4, 2, 128, 16, seed=15)
    q, hint = _rows_and_hint(s, new)
    k, v, tab, qs = dev_bf16(s.k), dev_bf16(s.v), dev_i32(s.table), dev_i32(s.q_start)
    kv = dev_i32(s.kv)
    O = torch.empty_like(q)
    ws = emb.paged_workspace()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with emb.Recording(stream, keep=[q, k, v, tab, qs, kv, O, ws]) as rec:
        emb.emb_paged_attention(q, k, v, tab, qs, kv, O, s.scale, hint, ws, stream=stream)
    for lens in ([new + 600, new + 40], [new, new + 39], [new + 300, new]):
        s.kv = lens
        with torch.cuda.stream(stream):
            kv.copy_(dev_i32(lens))
            rec.launch(stream)
        torch.cuda.synchronize()
        assert torch.equal(O[:s.T], s.run())
    rec.close()


def test_on_another_stream_than_the_current(cuda_device):
    s = Paged([1, 70], [500, 300], 8, 2, 128, 16, seed=16)
    assert torch.equal(s.run(), s.run(stream=torch.cuda.Stream()))


@pytest.mark.parametrize("new", [1, 100])
def test_cache_beyond_32_bits(cuda_device, new):
    """Pages whose byte and element offsets pass 2^32."""
    Hk, d, page = 8, 128, 64
    n_pages = (1 << 33) // (page * Hk * d)  # 2^33 elements
    s = Paged([new], [new + 200], Hk, Hk, d, page, seed=17)
    n = s.table.shape[1]
    kc = torch.zeros(n_pages, page, Hk, d, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros(n_pages, page, Hk, d, dtype=torch.bfloat16, device="cuda")
    far = np.array([[n_pages - 1 - 3 * i for i in range(n)]])
    for i in range(n):
        kc[far[0, i]], vc[far[0, i]] = dev_bf16(s.k[s.table[0, i]]), dev_bf16(s.v[s.table[0, i]])
    q, hint = _rows_and_hint(s, new)
    O = torch.empty_like(q)
    emb.emb_paged_attention(q, kc, vc, dev_i32(far), dev_i32(s.q_start), dev_i32(s.kv), O, s.scale, hint,
                            emb.paged_workspace())
    assert torch.equal(O[:s.T], s.run())
    # and the cache write reaches them
    slots = torch.tensor([(n_pages - 1) * page + 7], dtype=torch.int64, device="cuda")
    x = torch.randn(1, Hk * d, device="cuda").to(torch.bfloat16)
    emb.emb_qk_norm_rope(x, x, x, torch.empty_like(x), kc, vc, slots, torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert torch.equal(vc[n_pages - 1, 7].view(-1), x[0]) and torch.equal(kc[n_pages - 1, 7].view(-1), x[0])
