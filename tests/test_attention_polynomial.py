"""The polynomial that stands for tanh in capped scores of bf16 queries: its error is what the comment beside it says, and no polynomial of that form does better by more than rounding."""
import os
import re

import numpy as np

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2401_15077_amd", "csrc", "chunk_attn.h")


def coefficients():
    text = open(SOURCE).read()
    body = text[text.index("auto bent"):]
    body = body[:body.index("return x * fmaf(t, z, k);")]
    a4, a3, a2, a1 = (float(x) for x in re.findall(r"k \* (-?[0-9.]+)f", body))
    said = re.search(r"up to ([0-9.]+), which is ([0-9.]+) \* 10\^-([0-9]+)", body)
    return [a1, a2, a3, a4], float(said[1]), float(said[2]) * 10.0 ** -int(said[3])


def test_its_error_is_what_its_comment_says():
    a, end, said = coefficients()
    y = np.linspace(0.0, end, 400001)
    z = y * y
    p = y * (1 + z * (a[0] + z * (a[1] + z * (a[2] + z * a[3]))))
    worst = np.abs(p - np.tanh(y)).max()
    assert said * 0.98 <= worst <= said * 1.01, worst


def test_no_other_polynomial_of_its_form_is_better():
    """Alternation: the error reaches its largest size five times, with signs in turn (four coefficients are free), so any other polynomial of the form is off by as much at one of those places."""
    a, end, said = coefficients()
    y = np.linspace(0.0, end, 400001)
    z = y * y
    e = y * (1 + z * (a[0] + z * (a[1] + z * (a[2] + z * a[3])))) - np.tanh(y)
    tops, sign = [], 0
    for x in e[np.abs(e) > 0.97 * said]:
        if np.sign(x) != sign:
            tops.append(x)
            sign = np.sign(x)
    assert len(tops) >= 5, tops
