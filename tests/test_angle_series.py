"""The series that angles of the append to 8-bit codes are worked out by: the coefficients are the factorials', and what is left out is what the comment beside them says."""
import math
import os
import re
from fractions import Fraction

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2401_15077_amd", "csrc", "rope_coded.h")


def parts():
    text = open(SOURCE).read()
    said = text[text.index("// Cosine and sine of position"):]
    body = said[said.index("cos_sin_turn64"):]
    said, body = said[:said.index("__device__")], body[:body.index("return")]
    number = r"(-?[0-9.]+(?:e-?[0-9]+)?)"
    s = [re.search(r"double s = " + number, body)[1]] + re.findall(r"s = fma\(s, z, " + number, body)
    c = [re.search(r", c = " + number, body)[1]] + re.findall(r"c = fma\(c, z, " + number, body)
    return said, [float(x) for x in reversed(s)], [float(x) for x in reversed(c)]


def test_the_coefficients():
    _, s, c = parts()
    assert s == [float(Fraction((-1) ** k, math.factorial(2 * k + 1))) for k in range(1, len(s) + 1)]
    assert c == [float(Fraction((-1) ** k, math.factorial(2 * k))) for k in range(len(c))]


def test_what_is_left_out():
    """Terms alternate and fall, so what is left out is less than the first term of it, and more than that less the next."""
    said, s, c = parts()
    sine, cosine = (Fraction(1, 2 ** int(n)) for n in re.search(r"less than 2\^-(\d+) of a sine and 2\^-(\d+) of a\s+// cosine", said).groups())
    x = Fraction(math.pi / 4) + Fraction(1, 2 ** 50)
    for first, bound in ((2 * len(s) + 3, sine), (2 * len(c), cosine)):
        term = x ** first / math.factorial(first)
        assert term < bound < 2 * term, (first, float(term), float(bound))


def test_a_turn():
    text = open(SOURCE).read()
    assert float(re.search(r"\* ([0-9.]+e-[0-9]+);\s+// 2 pi / 2\^64", text)[1]) == 2 * math.pi / 2 ** 64
