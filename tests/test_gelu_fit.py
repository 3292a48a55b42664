"""The gated block's fit to gelu's tail: its stated error, with the constants that the source holds."""
import os
import re

import numpy as np
from scipy.special import erfcx

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2212_11142_amd", "csrc")


def test_stated_error():
    text = open(os.path.join(CSRC, "gated.hip")).read()
    slope = float(np.float32(re.search(r"rcpf\(fmaf\(([0-9.]+)f, fabsf\(z\)", text).group(1)))
    body = text[text.index("float q = -0.5f"):text.index("const float e = fast_exp2(z * z")]
    fit = [float(s + "0.5") * float(np.float32(c)) for s, c in re.findall(r"(-?)0\.5f \* ([0-9.]+)f", body)]
    assert len(fit) == 7
    stated = float(re.search(r"relative error of ([0-9.e-]+) up to \|z\| = ([0-9.]+)", text).group(1))
    z = np.concatenate([np.linspace(0, 14.5, 400001), np.logspace(-9, 0, 10001)])
    t, q = 1 / (1 + slope * z), 0.0
    for c in fit:
        q = q * t + c
    off = np.abs(q / (0.5 * erfcx(z / np.sqrt(2)) / t) - 1).max()
    assert off <= stated < 1.02 * off
