"""The constants that angles of the append to 8-bit codes are worked out by."""
import math
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2401_15077_amd", "csrc", "rope_coded.h")


def test_a_turn():
    text = open(SOURCE).read()
    assert float(re.search(r"\* ([0-9.]+e-[0-9]+);\s+// 2 pi / 2\^64", text)[1]) == 2 * math.pi / 2 ** 64
