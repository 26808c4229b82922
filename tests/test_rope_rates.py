"""The rates of rotary positions against 40-digit arithmetic, at the bound that the header gives (CPU only)."""
import ctypes
import decimal
import math

import pytest

from paper_2602_07160_gb300 import build, fem

D = decimal.Decimal
PI = D("3.14159265358979323846264338327950288419716939937510582097494459")
CONTEXT, LOW, HIGH = 4096.0, 1.0, 32.0


@pytest.fixture(scope="module")
def lib():
    build.build()
    return fem.load()


def some(table):
    """Up to some 40 pairs of a table, the first and last among them."""
    n = len(table)
    return [(i, table[i]) for i in sorted({*range(0, n, 1 + n // 40), n - 1})]


def power(base, exponent):
    return (base.ln() * exponent).exp()


@pytest.mark.parametrize("base", [0.5, 1.0, 10.0, 500.0, 1e4, 5e5, 1e6, 1e9])
@pytest.mark.parametrize("scaling,factor", [(None, 1.0), ("linear", 8.0), ("linear", 0.125), ("linear", 3.0), ("base", 8.0), ("base", 1000.0),
                                            ("parts", 8.0), ("parts", 0.3)])
def test_rates_are_off_by_no_more_than_stated(lib, base, scaling, factor):
    with decimal.localcontext() as context:
        context.prec = 40
        for rotary in (2, 4, 6, 20, 74, 128, 256, 1024):
            table = (ctypes.c_uint64 * (rotary // 2))()
            assert lib.fem_rope_turns(rotary, base, fem.Rope.SCALINGS[scaling], factor, CONTEXT, LOW, HIGH, table) == 0
            b, f = D(base), D(factor)
            if scaling == "base" and rotary > 2:
                b *= power(f, D(rotary) / (rotary - 2))
            for i, got in some(table):
                rate = power(b, D(-2 * i) / rotary)
                off = (7 + abs(math.log(base)) + 4 * abs(math.log(factor))) * 2.0 ** -53  # of the rate
                if scaling == "linear":
                    rate /= f
                if scaling == "parts":
                    c = D(CONTEXT) * rate / (2 * PI)
                    g = min(D(1), max(D(0), (c - D(LOW)) / D(HIGH - LOW)))
                    rate = g * rate + (1 - g) * rate / f
                    if 0 < g < 1:  # and g's part, off by its numerator's roundings
                        off *= 1 + 2 * float(c) / (HIGH - LOW) * max(1.0, 1 / factor) / (float(g) + (1 - float(g)) / factor)
                turn = rate / (2 * PI)
                error = abs(D(got) / D(2) ** 64 - turn % 1)
                error = min(error, 1 - error)
                assert error <= D(off) * turn + D(2) ** -64, (rotary, i, float(error / turn) * 2.0 ** 53, off * 2.0 ** 53)


def test_plain_rates_are_good_for_positions_to_2_27(lib):
    """For bases of at least 1 a position's angle is off by less than 3 2^-53 rad a position, fp32's rounding of 1 at 2^27 and more."""
    with decimal.localcontext() as context:
        context.prec = 40
        for base in (1.0, 2.0, 500.0, 1e4, 5e5, 1e6, 1e9):
            for rotary in (6, 74, 96, 128, 1024):
                table = (ctypes.c_uint64 * (rotary // 2))()
                assert lib.fem_rope_turns(rotary, base, 0, 1.0, 0.0, 0.0, 0.0, table) == 0
                for i, got in some(table):
                    turn = power(D(base), D(-2 * i) / rotary) / (2 * PI)
                    assert abs(D(got) / D(2) ** 64 - turn) * 2 * PI <= D(3) * D(2) ** -53
