"""emb_paged8_store and emb_paged8_read against the oracle: values and untouched keys bit for bit, normalised and rotated ones
within the bound of fp32 and one rounding; blocks begun, gone on with, grown and left alone; every head size and layout."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_02501_gb300 as emb
from tests.paged_util import dev_bf16, dev_i32, host
from tests.paged8_util import dev_u8

pytestmark = pytest.mark.gpu
BLOCK = 16


def dev_i64(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(np.int64))).cuda()


def same_values(a, b):
    return np.array_equal(a, b, equal_nan=True)


class Step:
    """A cache of random codes and exponents, and the tokens of a step: requests with cached[r] tokens and new[r] more, whose pages lie
    in random order."""

    def __init__(self, cached, new, H, Hk, d, page, seed, gain=1.0):
        rng = np.random.default_rng(seed)
        self.rng, self.H, self.Hk, self.d, self.page = rng, H, Hk, d, page
        pages = [-(-(c + n) // page) for c, n in zip(cached, new)]
        self.n_pages = sum(pages) + 2
        perm, at, slots, pos = rng.permutation(self.n_pages), 0, [], []
        for c, n, k in zip(cached, new, pages):
            mine = perm[at:at + k]
            at += k
            slots += [int(mine[p // page]) * page + p % page for p in range(c, c + n)]
            pos += list(range(c, c + n))
        self.slots, self.positions, self.T = np.array(slots, dtype=np.int64), np.array([pos], dtype=np.int64), len(slots)
        shape = (self.n_pages, page, Hk, d)
        self.codes = [rng.integers(0, 256, shape).astype(np.uint8) for _ in range(2)]
        self.exps = [rng.integers(118, 124, (self.n_pages, page // BLOCK, Hk)).astype(np.uint8) for _ in range(2)]
        draw = lambda w: oracle.bf16_round(rng.standard_normal((self.T, w * d)) * gain)
        self.q, self.k, self.v = draw(H), draw(Hk), draw(Hk)
        self.q_gamma = self.k_gamma = self.axis = None
        self.turns, self.neighbours, self.factor, self.eps = [], False, 1.0, 1e-6

    def rotate(self, rot, neighbours=False, axes=1, **kw):
        self.turns = [int(t) % 2 ** 64 for t in emb.emb_rotary_turns(rot, **kw).tolist()]
        self.neighbours = neighbours
        if axes > 1:
            self.positions = np.concatenate([self.positions] + [self.rng.integers(-50, 5000, self.positions.shape) for _ in range(axes - 1)])
            self.axis = self.rng.integers(0, axes, rot // 2)
        return self

    def norm(self):
        self.q_gamma, self.k_gamma = (1 + 0.1 * self.rng.standard_normal((2, self.d))).astype(np.float32)
        return self

    def device(self):
        f32 = lambda x: None if x is None else torch.from_numpy(x).cuda()
        self.cache = [dev_u8(x) for x in self.codes + self.exps]
        self.q_out = torch.full((self.T, self.H * self.d), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.args = [dev_bf16(self.q), dev_bf16(self.k), dev_bf16(self.v), self.q_out, *self.cache, dev_i64(self.slots), dev_i32(self.positions),
                     dev_i64(np.array(self.turns, dtype=np.uint64).view(np.int64)) if len(self.turns) else None]
        self.kw = dict(q_gamma=f32(self.q_gamma), k_gamma=f32(self.k_gamma), eps=self.eps, neighbours=self.neighbours, factor=self.factor,
                       axis_of_pair=None if self.axis is None else dev_u8(self.axis))
        return self

    def rows(self, x, heads, gamma):
        axis = [0] * len(self.turns) if self.axis is None else self.axis
        return oracle.norm_turn_reference(x, heads, self.d, gamma, self.eps, self.positions, axis, self.turns, self.neighbours, self.factor)

    def check(self, what=""):
        """One call on copies of the cache against the oracle."""
        self.device()
        emb.emb_paged8_store(*self.args, **self.kw)
        torch.cuda.synchronize()
        kc, vc, ke, ve = [c.cpu().numpy() for c in self.cache]
        y, err = self.rows(self.q, self.H, self.q_gamma)
        out = host(self.q_out).reshape(y.shape)
        bad = np.abs(out - y) > oracle.bf16_bound(y, err)
        assert not bad.any() and np.isfinite(out).all(), f"{what}: {int(bad.sum())} queries off, first {np.argwhere(bad)[:3].tolist()}"
        want_c, want_e = oracle.paged8_store_reference(self.v.reshape(self.T, self.Hk, self.d).astype(np.float64), self.codes[1], self.exps[1], self.slots)
        assert np.array_equal(ve, want_e), what
        assert same_values(oracle.paged8_values(vc, ve), oracle.paged8_values(want_c, want_e)), what
        y, err = self.rows(self.k, self.Hk, self.k_gamma)
        if not err.any():
            want_c, want_e = oracle.paged8_store_reference(y, self.codes[0], self.exps[0], self.slots)
            assert np.array_equal(ke, want_e), what
            assert same_values(oracle.paged8_values(kc, ke), oracle.paged8_values(want_c, want_e)), what
            return self
        # exponents between those of the least and the most that the rows may be; codes within half a step of that
        lo_c, lo_e = oracle.paged8_store_reference(np.sign(y) * np.maximum(np.abs(y) - err, 0), self.codes[0], self.exps[0], self.slots)
        hi_c, hi_e = oracle.paged8_store_reference(y + np.sign(y) * err, self.codes[0], self.exps[0], self.slots)
        assert ((ke >= lo_e) & (ke <= hi_e)).all(), what
        got = oracle.paged8_values(kc, ke)
        ok = (self.slots >= 0) & (self.slots < self.n_pages * self.page)
        pg, at = self.slots[ok] // self.page, self.slots[ok] % self.page
        unit = 2.0 ** oracle.exponent_of(ke)[pg, at // BLOCK][..., None]
        off = np.abs(got[pg, at] - y[ok])
        assert (off <= err[ok] + np.maximum(2.0 ** -4 * (np.abs(y[ok]) + err[ok]), 2.0 ** -10 * unit)).all(), what
        same = np.repeat(lo_e == hi_e, BLOCK, axis=1)
        same[pg, at] = False
        assert same_values(got[same], oracle.paged8_values(lo_c, lo_e)[same]), what
        return self


SHAPES = [([0], [1]), ([866], [1]), ([0], [50]), ([7], [40]), ([0, 5, 31], [3, 11, 17]), ([15, 16, 17, 1], [1, 1, 1, 1]), ([3], [300]),
          ([2, 0, 9, 100], [20, 0, 7, 61]), (list(range(40)), [1] * 40), (list(range(0, 90, 3)), [5] * 30)]


@pytest.mark.parametrize("cached,new", SHAPES)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 32), (256, 64)])
def test_values_and_bare_keys_bit_for_bit(cuda_device, cached, new, d, page):
    for gain in (0.01, 1.0, 50.0):
        Step(cached, new, 4, 2, d, page, seed=sum(new) + d, gain=gain).check(f"gain {gain}")


@pytest.mark.parametrize("cached,new", SHAPES)
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 24), (128, 128), (128, 64), (256, 256), (256, 8)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_norm_and_rotation(cuda_device, cached, new, d, rot, neighbours):
    s = Step(cached, new, 6, 2, d, 16, seed=rot + sum(new)).norm().rotate(rot, neighbours, axes=1 + (rot > 24) * 2, base=10000.0)
    s.check()


@pytest.mark.parametrize("neighbours", [False, True])
def test_far_positions_stretched_and_scaled(cuda_device, neighbours):
    s = Step([0], [40], 3, 1, 128, 16, seed=3).rotate(128, neighbours, base=5e5, stretch=8.0, original=8192.0)
    s.factor = 1.25
    s.positions = s.rng.integers(-2 ** 31, 2 ** 31, s.positions.shape)
    s.check()
    s.positions[:] = 2 ** 31 - 1
    s.check()
    s.factor = 0.0
    s.check()


def test_heads_of_all_counts(cuda_device):
    for H, Hk in ((1, 1), (5, 5), (64, 1), (7, 1), (28, 4), (3, 9), (100, 2)):
        Step([9, 30], [9, 30], H, Hk, 64, 16, seed=H).norm().rotate(64).check(f"{H} on {Hk}")


def test_strided_rows(cuda_device):
    """A packed projection's rows."""
    s = Step([3], [37], 4, 2, 128, 16, seed=5).norm().rotate(64, True).device()
    T, d = s.T, s.d
    packed = torch.full((T, (4 + 2 + 2 + 1) * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    parts = packed[:, :8 * d].split([4 * d, 2 * d, 2 * d], dim=1)
    for to, x in zip(parts, s.args[:3]):
        to.copy_(x)
    emb.emb_paged8_store(*s.args, **s.kw)
    want = [x.clone() for x in [s.q_out] + s.cache]
    s.device()
    emb.emb_paged8_store(*parts, *s.args[3:], **s.kw)
    assert all(torch.equal(a, b) for a, b in zip(want, [s.q_out] + s.cache))


def test_tokens_without_a_slot(cuda_device):
    """Slots below 0 or beyond the cache: queries only; the tokens on both sides are stored as if they were not there."""
    s = Step([4], [40], 2, 2, 64, 16, seed=6).norm().rotate(64)
    s.slots[[0, 7, 20, 21, 39]] = [-1, s.n_pages * s.page, -2 ** 40, 2 ** 62, -1]
    s.check()
    s.slots[:] = -1
    s.check()
    assert all(np.array_equal(c.cpu().numpy(), w) for c, w in zip(s.cache, s.codes + s.exps))


def test_odd_values(cuda_device):
    """NaN, infinities and what is above the largest exponent become NaN codes and do not count for the exponent; zeros, the smallest
    numbers and the largest that there is room for."""
    s = Step([0], [16 * 6], 1, 1, 64, 16, seed=7)
    for x in (s.k, s.v):
        x[0:16, 3] = np.nan
        x[16, 5], x[17, 6] = np.inf, -np.inf
        x[32:48] = 0.0
        x[48:64] = oracle.bf16_round(x[48:64] * 1e-30)
        x[64] = oracle.bf16_round(448.0 * 2.0 ** 48)
        x[65] = -x[64]
        x[80] = 3e38
        x[81] = oracle.bf16_round(450.0 * 2.0 ** 48)
    s.q[3], s.q[5] = np.nan, np.inf
    s.device()
    emb.emb_paged8_store(*s.args, **s.kw)
    kc, vc, ke, ve = [c.cpu().numpy() for c in s.cache]
    for x, c, e, i in ((s.k, kc, ke, 0), (s.v, vc, ve, 1)):
        want_c, want_e = oracle.paged8_store_reference(x.reshape(-1, 1, 64).astype(np.float64), s.codes[i], s.exps[i], s.slots)
        assert np.array_equal(e, want_e)
        assert same_values(oracle.paged8_values(c, e), oracle.paged8_values(want_c, want_e))
        pg, at = s.slots // 16, s.slots % 16
        assert np.isnan(oracle.paged8_values(c, e)[pg[80:82], at[80:82]]).all() and ve.max() <= 127 + 48
    out = host(s.q_out)
    assert np.isnan(out[3]).all() and np.isinf(out[5]).all() and np.isfinite(np.delete(out, [3, 5], axis=0)).all()


def test_grows_and_keeps(cuda_device):
    """Token by token into one block: small values first, then larger ones; what was there keeps its values to the new unit, twice the same
    call changes nothing, and the first place starts the block anew."""
    s = Step([0], [16], 1, 1, 128, 16, seed=8)
    s.v *= 2.0 ** np.arange(-6, 10)[:, None]
    s.v = oracle.bf16_round(s.v)
    s.device()
    q, k, v = s.args[:3]
    for t in list(range(16)) + [0, 5]:
        one = [x[t:t + 1] for x in (q, k, v, s.q_out)]
        codes, exps = s.cache[1].cpu().numpy(), s.cache[3].cpu().numpy()
        for _ in range(2):
            emb.emb_paged8_store(*one, *s.cache, s.args[8][t:t + 1], s.args[9][:, t:t + 1], None)
            want_c, want_e = oracle.paged8_store_reference(s.v[t:t + 1].reshape(1, 1, 128), codes, exps, s.slots[t:t + 1])
            got_c, got_e = s.cache[1].cpu().numpy(), s.cache[3].cpu().numpy()
            assert np.array_equal(got_e, want_e) and same_values(oracle.paged8_values(got_c, got_e), oracle.paged8_values(want_c, want_e)), t


def test_one_call_or_token_by_token(cuda_device):
    """Normal codes do not depend on how the tokens came: a power of two moves no mantissa bits."""
    s = Step([0], [64], 1, 2, 64, 32, seed=9)
    s.device()
    emb.emb_paged8_store(*s.args, **s.kw)
    slots = s.args[8]
    whole = [torch.empty(64, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    emb.emb_paged8_read(*s.cache, slots, *whole)
    exps = [c.clone() for c in s.cache[2:]]
    q, k, v = s.args[:3]
    s.cache = [dev_u8(x) for x in s.codes + s.exps]
    for t in range(64):
        emb.emb_paged8_store(q[t:t + 1], k[t:t + 1], v[t:t + 1], s.q_out[t:t + 1], *s.cache, slots[t:t + 1], s.args[9][:, t:t + 1], None)
    single = [torch.empty_like(x) for x in whole]
    emb.emb_paged8_read(*s.cache, slots, *single)
    pg, blk = s.slots // 32, s.slots % 32 // 16
    for a, b, e, f in zip(whole, single, exps, s.cache[2:]):
        assert torch.equal(e[pg, blk], f[pg, blk])
        unit = torch.exp2(e[pg, blk].float() - 127).repeat_interleave(64, 1)
        normal = a.float().abs() >= 2.0 ** -6 * unit
        assert torch.equal(a[normal], b[normal]) and ((a.float() - b.float()).abs() <= 2.0 ** -9 * unit)[~normal].all()


@pytest.mark.parametrize("d,page,Hk", [(64, 16, 1), (128, 64, 8), (256, 256, 3), (64, 128, 70)])
@pytest.mark.parametrize("n", [1, 3, 1000])
def test_read(cuda_device, d, page, Hk, n):
    rng = np.random.default_rng(n)
    codes = [rng.integers(0, 256, (7, page, Hk, d)).astype(np.uint8) for _ in range(2)]
    exps = [rng.integers(0, 256, (7, page // BLOCK, Hk)).astype(np.uint8) for _ in range(2)]
    slots = rng.integers(-5, 7 * page + 5, n)
    slots[0] = 7 * page - 1
    out = [torch.full((n + 2, Hk * d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    emb.emb_paged8_read(*map(dev_u8, codes + exps), dev_i64(slots), *(o[:n] for o in out))
    ok = (slots >= 0) & (slots < 7 * page)
    at = np.where(ok, slots, 0)
    for o, c, e in zip(out, codes, exps):
        want = np.where(ok[:, None], oracle.paged8_values(c, e)[at // page, at % page].reshape(n, -1), 0.0)
        assert same_values(host(o)[:n], want) and (host(o)[n:] == 7).all()


def test_read_nothing(cuda_device):
    cache = emb.paged8_cache(2, 16, 1, 64)
    none = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    emb.emb_paged8_read(*cache, torch.empty(0, dtype=torch.int64, device="cuda"), none, none.clone())


def test_recorded_and_on_another_stream(cuda_device):
    """A recorded store follows slots, positions and rows from replay to replay."""
    s = Step([5, 30], [11, 9], 4, 2, 128, 16, seed=10).norm().rotate(128).device()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with emb.Recording(stream, keep=[s.args, s.kw]) as rec:
        emb.emb_paged8_store(*s.args, **s.kw, stream=stream)
    for seed in (11, 12):
        n = Step([5, 30], [11, 9], 4, 2, 128, 16, seed=seed).norm().rotate(128)
        n.k_gamma, n.q_gamma = s.k_gamma, s.q_gamma
        n.device()
        emb.emb_paged8_store(*n.args, **n.kw)
        want = [x.clone() for x in [n.q_out] + n.cache]
        n.device()
        with torch.cuda.stream(stream):
            for to, x in zip(s.args[:3] + s.cache + s.args[8:10], n.args[:3] + n.cache + n.args[8:10]):
                to.copy_(x)
            rec.launch(stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [s.q_out] + s.cache))
    rec.close()


def test_tokens_of_a_block_in_any_order(cuda_device):
    """Within 16 consecutive tokens: each block's tokens backwards, and two blocks' tokens in turns."""
    s = Step([5, 0], [60, 40], 2, 2, 128, 32, seed=13).norm().rotate(64)
    order, blocks = [], s.slots // BLOCK
    for b in dict.fromkeys(blocks.tolist()):
        order += np.flatnonzero(blocks == b)[::-1].tolist()
    s.slots, s.positions = s.slots[order], s.positions[:, order]
    s.check("backwards")
    s = Step([9, 9], [7, 7], 2, 1, 64, 16, seed=14)
    order = np.arange(14).reshape(2, 7).T.reshape(-1)
    s.slots, s.positions = s.slots[order], s.positions[:, order]
    s.check("in turns")


def test_positions_wider_than_the_tokens(cuda_device):
    """Positions of several axes cut out of a wider table."""
    s = Step([3], [21], 2, 1, 64, 16, seed=15).rotate(64, axes=3).device()
    emb.emb_paged8_store(*s.args, **s.kw)
    want = [x.clone() for x in [s.q_out] + s.cache]
    s.device()
    wide = torch.full((3, 50), 10 ** 6, dtype=torch.int32, device="cuda")
    wide[:, :s.T] = s.args[9]
    emb.emb_paged8_store(*s.args[:9], wide, *s.args[10:], **s.kw)
    assert all(torch.equal(a, b) for a, b in zip(want, [s.q_out] + s.cache))
