"""Angles of far positions: the kernels' own arithmetic, compiled on its own, against exact arithmetic (no GPU needed)."""
import math
import random
import struct
from fractions import Fraction

from test_host_kv_rules import _run

PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798214808651")


def test_a_turn_is_off_by_the_rounding_to_fp32_whatever_the_position(tmp_path):
    """The part of a turn is below 1: its rounding to fp32 is off by 2^-25 at most.  Position times frequency and 1 / (2 pi) take two
    64-bit words each, so what they lose, 2^-100 of the turns, is nothing for up to 2^51 of them (allowed: a millionth of the rounding)."""
    r = random.Random(7)
    cases = [(p, f) for p in (0, 1, -1, 35, 900000, -(1 << 31), (1 << 31) - 1, (1 << 24) + 1) for f in (1.0, 0.5, 1e-6, 0.9306, 1e4 ** (-1 / 64))]
    cases += [(r.randint(1 << 30, (1 << 31) - 1) * r.choice((1, -1)), r.uniform(0.5, 1.0)) for _ in range(4000)]
    cases += [(r.randint(-(1 << 31), (1 << 31) - 1), 2.0 ** r.uniform(-40, 20)) for _ in range(4000)]
    rows = []
    for p, f in cases:
        bits = struct.unpack("<I", struct.pack("<f", f))[0]
        turns = p * Fraction(struct.unpack("<f", struct.pack("<f", f))[0]) / (2 * PI)
        part = turns - round(turns)
        hi = float(part)
        rows.append("{%dll, %du, %s, %s}" % (p, bits, hi.hex(), float(part - Fraction(hi)).hex()))
    _run(tmp_path, r"""
    struct Case { long long p; unsigned f; double part, rest; };
    static const Case cases[] = {%s};
    for (const Case &c : cases) {
        float f;
        __builtin_memcpy(&f, &c.f, 4);
        double off = ((double)part_of_turn((int)c.p, f) - c.part) - c.rest;
        off -= rint(off);                                       // (half a turn either way is the same)
        if (!(std::fabs(off) <= %s)) return 1;
    }""" % (",\n".join(rows), (2.0 ** -25 * (1 + 1e-6)).hex()), "turns.h")
    assert math.isclose(float(PI), math.pi)
