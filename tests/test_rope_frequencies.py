"""The frequencies of rotary positions (pe_rope_init) against numbers of 60 digits (no GPU needed)."""
from decimal import Decimal, localcontext

import pytest

from paper_2509_04377_amd import binding as pe

TWO_PI = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


def _turns(R, base, scaling, factor, low, high, original):
    """f_i / 2 pi in units of 2^-64 turns, with what a double stands for taken at its word."""
    with localcontext() as c:
        c.prec = 60
        ln = Decimal(base).ln()
        for i in range(R // 2):
            f = (-2 * Decimal(i) / R * ln).exp()
            if scaling == pe.PE_ROPE_LINEAR:
                f /= Decimal(factor)
            elif scaling == pe.PE_ROPE_BY_PARTS:
                g = (Decimal(original) * f / TWO_PI - Decimal(low)) / (Decimal(high) - Decimal(low))
                g = min(Decimal(1), max(Decimal(0), g))
                f *= g + (1 - g) / Decimal(factor)
            yield f / TWO_PI * 2 ** 64


@pytest.mark.parametrize("R", [2, 6, 40, 64, 126, 128])
@pytest.mark.parametrize("base", [1.5, 1e4, 10007.3, 5e5, 1e6, 1e15])
@pytest.mark.parametrize("scaling,kw", [(pe.PE_ROPE_PLAIN, {}), (pe.PE_ROPE_LINEAR, dict(factor=4.0)), (pe.PE_ROPE_LINEAR, dict(factor=2.3)),
                                        (pe.PE_ROPE_BY_PARTS, dict(factor=8.0, low=1.0, high=4.0, original=8192.0)),
                                        (pe.PE_ROPE_BY_PARTS, dict(factor=32.0, low=0.0, high=3.7, original=5000.5)),
                                        (pe.PE_ROPE_BY_PARTS, dict(factor=3.0, low=1.0, high=64.0, original=100.0))])
def test_within_two_units(R, base, scaling, kw):
    a = dict(factor=1.0, low=1.0, high=4.0, original=8192.0)
    a.update(kw)
    rope = pe.make_rope(R, base, scaling=scaling, **kw)
    off = [abs(rope.turns[i] - t) for i, t in enumerate(_turns(R, base, scaling, **a))]
    assert len(off) == R // 2 and max(off) <= 2, max(off)
    assert list(rope.turns)[R // 2:] == [0] * (64 - R // 2)
