"""The fit behind the gated layer's normal distribution, from the constants in the source, against 64 bits (no GPU).

Below -x the distribution is exp(-x^2/2) R(x), and R(x) = exp(x^2/2) erfc(x / sqrt 2) / 2 = erfcx(x / sqrt 2) / 2, which scipy gives to some 1e-16."""
import os
import re

import numpy as np
from scipy.special import erfcx

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2305_03152_amd", "csrc", "spp_hidden.h")


def _fit():
    """(what x is multiplied by, coefficients from the highest power down, the error that the comment states), as fp32 has the constants."""
    text = open(SOURCE).read()
    at = text.index("float normal(")
    body, comment = text[at:text.index("\n}", at)], text[text.rindex("\n\n", 0, at):at]
    slope = re.search(r"__fmaf_rn\(([\d.]+)f, x, 1\.0f\)", body).group(1)
    first = re.search(r"float p = (-?[\d.]+)f;", body).group(1)
    rest = re.findall(r"__fmaf_rn\(p, t, (-?[\d.]+)f\)", body)
    stated = re.search(r"in fp32, ([\d.]+e-\d+)", comment).group(1)
    return float(np.float32(slope)), [float(np.float32(c)) for c in [first] + rest], float(stated)


def test_the_fit_is_as_near_as_its_comment_says():
    slope, coefficients, stated = _fit()
    assert len(coefficients) == 9
    x = np.linspace(0.0, 14.0, 1_400_001)
    t = 1 / (1 + slope * x)
    p = np.zeros_like(x)
    for c in coefficients:
        p = p * t + c
    off = np.abs(t * p / (erfcx(x / np.sqrt(2.0)) / 2) - 1).max()
    assert 0.9 * stated < off <= stated
