"""The rotary frequencies of w8a8_rope_frequencies against 60-digit arithmetic: how far a table's fractions of a turn are off,
which is what far positions multiply."""
from decimal import Decimal, getcontext

import pytest

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("linear", 0.25)])
@pytest.mark.parametrize("base", [1.5, 1e4, 5e5, 1e6, 1e8])
@pytest.mark.parametrize("rot", [16, 48, 64, 128, 208, 256])
def test_fractions_of_a_turn(B, rot, base, scaling, factor):
    """A double's quotient of a double's power: the power is off by 2^-52 of itself and by ln(base) times the half step its
    exponent is rounded by (2^-54 at most); the scaling, 2 pi and the quotient by 2^-53 each; the fraction is cut at 2^-64."""
    getcontext().prec = 60
    turns, _ = B.rope_frequencies(B.RopeConfig(rot, base=base, scaling=scaling, factor=factor))
    ln = Decimal(base).ln()
    for i, t in enumerate(turns.tolist()):
        f = (-ln * 2 * i / rot).exp() / Decimal(factor)
        want = f / (2 * PI) % 1
        got = Decimal(t % (1 << 64)) / (1 << 64)
        off = abs(got - want)
        bound = f / (2 * PI) * (Decimal(2) ** -52 + ln * Decimal(2) ** -54 + 3 * Decimal(2) ** -53) + Decimal(2) ** -64
        assert min(off, 1 - off) <= bound, (i, float(off / bound))


@pytest.mark.parametrize("factor", [1e-6, 4.5e-5, 0.25, 0.9999, 1.0, 1.0001, 16.0])
def test_parts_by_a_factor_of_one_or_less(B, factor):
    """The factor on cos and sin that PARTS brings with it is 1 where positions are not compressed: never below, let alone
    zero or negative (0.1 ln(factor) + 1 is at factors of e^-10 and less)."""
    import math
    from oracle import serving as OS
    kw = dict(factor=factor, low=1.0, high=32.0, original_len=4096)
    _, scale = B.rope_frequencies(B.RopeConfig(64, scaling="parts", **kw))
    want = 1.0 + max(0.0, 0.1 * math.log(factor))
    assert abs(scale - want) <= 2.0 ** -24 * want
    assert OS.rope_frequencies(64, 1e4, "parts", **kw)[1] == pytest.approx(want, abs=0, rel=2.0 ** -52)
    assert B.rope_frequencies(B.RopeConfig(64, scaling="parts", attn_factor=0.5, **kw))[1] == 0.5  # given, it is taken
