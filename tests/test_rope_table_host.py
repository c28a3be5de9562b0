"""How far the rotation's table is off, without a GPU: the part of an angle's error that grows with the position.

An entry is f / 2 pi with f = base^(-x), x = 2i / rot_dim, in 64-bit floats (a unit is 2^-52 of a value, a rounding half
of that): the power is off by a unit at most and by the exponent's rounding, 2^-53 x ln(base) of itself, 2 pi and the
quotient by half a unit each.  f <= 1 and f x ln(base) <= 1/e, so that in turns
  (2^-52 + 2^-53 + 2^-53 + 2^-53 / e) / 2 pi < 2^-53.
"""
import decimal

import pytest

PI2 = decimal.Decimal("6.28318530717958647692528676655900576839433879875021164194988918461563")


@pytest.fixture(scope="module")
def cure():
    import __graft_entry__
    try:
        __graft_entry__.build()
    except RuntimeError as e:  # no toolkit on this machine
        pytest.skip(f"cannot build libcure: {e}")
    from paper_2608_00531_gb300 import cure as c
    return c


@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.0e6])
def test_table(cure, base):
    worst = 0
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        for rot in (16, 96, 128):
            r = cure.rope_desc(rot, base)
            for i in range(rot // 2):
                want = decimal.Decimal(base) ** (decimal.Decimal(-2 * i) / rot) / PI2
                worst = max(worst, abs(decimal.Decimal(r.turns[i]) / 2 ** 64 - want))
    # (not closer than 2^-60 either: the entries hold 53 bits)
    assert decimal.Decimal(2.0 ** -60) < worst < decimal.Decimal(2.0 ** -53), float(worst)
