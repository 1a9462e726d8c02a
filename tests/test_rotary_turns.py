"""emb_rotary_turns against its formula in 80 digits: every pair within one unit of 2^-64 of a turn, whatever the base (CPU only)."""
from decimal import ROUND_FLOOR, Decimal, localcontext

import pytest

import paper_2607_02501_gb300 as emb

TWO_PI = 2 * Decimal("3.1415926535897932384626433832795028841971693993751058209749445923078164062862089986280348253421170679821")


def exact_units(rot_dim, base, stretch=1.0, original=0.0, low=1.0, high=32.0):
    """The turns per position in units of 2^-64, modulo one turn, not rounded."""
    out = []
    with localcontext() as c:
        c.prec = 80
        for i in range(rot_dim // 2):
            f = Decimal(base) ** (Decimal(-2 * i) / rot_dim)
            k = Decimal(0)
            if original > 0:
                k = (Decimal(original) * f / TWO_PI - Decimal(low)) / (Decimal(high) - Decimal(low))
                k = min(Decimal(1), max(Decimal(0), k))
            t = f * (k + (1 - k) / Decimal(stretch)) / TWO_PI
            out.append((t - t.to_integral_value(ROUND_FLOOR)) * 2 ** 64)
    return out


@pytest.mark.parametrize("rot_dim", [2, 6, 64, 96, 128, 250, 256])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1e6, 1.0, 3.7, 2.0 ** 40, 1e300, 0.5, 1e-4, 1e-8])
@pytest.mark.parametrize("long", [{}, {"stretch": 4.0}, {"stretch": 8.0, "original": 8192.0}, {"stretch": 32.1, "original": 1000.0, "low": 0.3, "high": 3.7},
                                  {"stretch": 2.0, "original": 1e300}, {"stretch": 2.0, "original": 1e-300, "low": 0.0}])
def test_turns_are_those_of_the_formula(rot_dim, base, long):
    got = [int(t) % 2 ** 64 for t in emb.emb_rotary_turns(rot_dim, base, **long).tolist()]
    want = exact_units(rot_dim, base, **long)
    off = [abs((Decimal(g) - w + 2 ** 63) % 2 ** 64 - 2 ** 63) for g, w in zip(got, want)]
    assert len(got) == rot_dim // 2 and max(off) <= 1, (max(off), off.index(max(off)))


@pytest.mark.parametrize("rot_dim", [258, 2 ** 40, 2 ** 62, -2 ** 62])
def test_sizes_beyond_a_head_are_refused(rot_dim):
    with pytest.raises(emb.EmbError) as e:
        emb.emb_rotary_turns(rot_dim)
    assert e.value.status == emb.EMB_EINVAL
