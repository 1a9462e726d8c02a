"""The 8-bit cache's oracle against independent statements of its format (CPU)."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2607_02501_gb300 as emb


def test_codes_are_torchs():
    """Values of all codes, and rounding at and around every border between two of them."""
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(oracle.e4m3_values(), want)
    v = oracle.e4m3_values()[:0x7F]
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), 0).astype(np.float64), np.nextafter(mid.astype(np.float32), 999).astype(np.float64)])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(oracle.e4m3_codes(x), want)


def test_rounding_error_is_half_a_step():
    x = np.random.default_rng(0).standard_normal(10000) * 30
    got = oracle.e4m3_values()[oracle.e4m3_codes(x)]
    assert (np.abs(got - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10)).all()


@pytest.mark.parametrize("top,e", [(0.0, -48), (448.0, 0), (np.nextafter(448.0, 999), 1), (3.5, -7), (3.6, -6), (449.0 * 2.0 ** 47, 48), (1e30, 48)])
def test_need(top, e):
    assert oracle.need_of(top) == e


def test_exponents_are_held_in_range():
    np.testing.assert_array_equal(oracle.exponent_of([0, 78, 79, 127, 175, 176, 255]), [-48, -48, -48, 0, 48, 48, 48])


def test_encode_and_values_round_trip():
    x = np.random.default_rng(1).standard_normal((3, 32, 2, 64)) * 10.0 ** np.arange(-3, 3).reshape(3, 1, 2, 1)
    codes, exps = oracle.paged8_encode(x)
    y = oracle.paged8_values(codes, exps)
    unit = 2.0 ** np.repeat(oracle.exponent_of(exps), 16, axis=1)[..., None]
    assert (np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * unit)).all()
    again = oracle.paged8_encode(y)
    np.testing.assert_array_equal(oracle.paged8_values(*again), y)


def test_store_by_hand():
    """One head, four dims' worth of cases: a block begun, one gone on with that has to grow, one that has not, and a token without a slot."""
    codes, exps = np.zeros((2, 32, 1, 64), dtype=np.uint8), np.full((2, 2, 1), 127, dtype=np.uint8)
    codes[0, 16:32] = oracle.e4m3_codes(1.0)         # block 1: ones
    codes[1, 16:32] = oracle.e4m3_codes(2.0 ** -9)   # block 3: the least there is
    rows = np.zeros((5, 1, 64))
    rows[0], rows[1], rows[2], rows[3], rows[4] = 0.75, 3.5, 7.0, 900.0, 1e9
    got, ex = oracle.paged8_store_reference(rows, codes, exps, [0, 1, 16 + 5, 32 + 16 + 3, -1])
    v = oracle.paged8_values(got, ex)[..., 0]
    assert ex[0, 0, 0] == 127 - 7 and (v[0, :2, 0] == [0.75, 3.5]).all() and (v[0, 2:16] == 0).all()
    assert ex[0, 1, 0] == 127 and v[0, 21, 0] == 7.0 and v[0, 22, 0] == 1.0
    assert ex[1, 1, 0] == 127 + 2 and v[1, 19, 0] == 896.0 and (v[1, 20:, 0] == 0).all()  # 2^-9 is a quarter of the new least
    assert ex[1, 0, 0] == 127 and (got[1, :16] == 0).all()


def test_turns():
    """The library's host function: radians a position in exact turns, stretched by parts."""
    for args in [dict(rot_dim=128), dict(rot_dim=64, base=5e5, stretch=8.0, original=8192.0), dict(rot_dim=32, stretch=4.0),
                 dict(rot_dim=256, base=0.5), dict(rot_dim=2)]:
        got = [int(t) % 2 ** 64 for t in emb.emb_rotary_turns(**args).tolist()]
        want = oracle.rotary_turns_reference(**{"base": 10000.0, **args})
        for g, w in zip(got, want):
            off = (g - w) % 2 ** 64
            # the formula's few roundings of fp64, relative to the frequency, of up to a few turns
            assert min(off, 2 ** 64 - off) <= 2 ** 64 * 2.0 ** -48, args
    f = [t / 2 ** 64 * 2 * math.pi for t in emb.emb_rotary_turns(8, 10000.0).tolist()]
    np.testing.assert_allclose(f, [1.0, 0.1, 0.01, 0.001], rtol=1e-12)
    s = [t / 2 ** 64 * 2 * math.pi for t in emb.emb_rotary_turns(8, 10000.0, 4.0).tolist()]
    np.testing.assert_allclose(s, np.array(f) / 4, rtol=1e-12)
    # pairs that turn 32 times in 1000 positions keep their rate, those that turn once or less are stretched
    p = [t / 2 ** 64 * 2 * math.pi for t in emb.emb_rotary_turns(8, 10000.0, 4.0, original=1000.0).tolist()]
    np.testing.assert_allclose([p[0], p[3]], [1.0, 0.00025], rtol=1e-12)
    assert 0.025 < p[1] < 0.1 and 0.0025 < p[2] < 0.01


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=258), dict(rot_dim=8, base=0.0), dict(rot_dim=8, base=float("nan")),
                                 dict(rot_dim=8, stretch=0.5), dict(rot_dim=8, original=-1.0), dict(rot_dim=8, low=2.0, high=2.0),
                                 dict(rot_dim=8, low=-1.0), dict(rot_dim=8, stretch=float("inf")), dict(rot_dim=-2)])
def test_turns_refusals(bad):
    with pytest.raises(emb.EmbError) as e:
        emb.emb_rotary_turns(**bad)
    assert e.value.status == emb.EMB_EINVAL


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation(neighbours):
    """Against the bf16 cache's oracle (halves), norms of pairs kept, and a turn that wraps exactly."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal((5, 2 * 64))
    turns = [int(t) % 2 ** 64 for t in emb.emb_rotary_turns(32).tolist()]
    pos = np.array([[0, 1, 77, 2 ** 20, -3]])
    y, err = oracle.norm_turn_reference(x, 2, 64, None, 0.0, pos, [0] * 16, turns, neighbours)
    if not neighbours:
        want, _ = oracle.qk_norm_rope_reference(x, 2, 64, None, 0.0, pos, [0] * 16, 32, 10000.0)
        np.testing.assert_allclose(y.reshape(5, -1), want, atol=1e-8)
    x3 = x.reshape(5, 2, 64)
    a, b = ([slice(0, 32, 2), slice(1, 32, 2)] if neighbours else [slice(0, 16), slice(16, 32)])
    np.testing.assert_allclose(y[..., a] ** 2 + y[..., b] ** 2, x3[..., a] ** 2 + x3[..., b] ** 2, rtol=1e-12)
    np.testing.assert_array_equal(y[..., 32:], x3[..., 32:])
    np.testing.assert_array_equal(y[0], x3[0])
    quarter, _ = oracle.norm_turn_reference(x, 2, 64, None, 0.0, np.full((1, 5), 2 ** 30 + 1), [0] * 4, [2 ** 62] * 4, neighbours)
    a, b = ([slice(0, 8, 2), slice(1, 8, 2)] if neighbours else [slice(0, 4), slice(4, 8)])
    np.testing.assert_allclose(quarter[..., a], -x3[..., b], atol=1e-12)
