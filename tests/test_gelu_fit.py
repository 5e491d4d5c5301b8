"""The coefficients of gelu's tail Q(a) = exp(-a^2 / 2) t S(t), t = 1 / (1 + 0.24 a), as the kernels have them, in 64 bits."""
import os
import re

import numpy as np
from scipy.special import erfcx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _coefficients():
    """S from its highest power down, and the 0.24, rounded to fp32 as the compiler rounds them."""
    text = open(os.path.join(ROOT, "paper_2007_13055_amd", "csrc", "bsr_epilogue.h")).read()
    body = text[text.index("void normal_tail("):]
    body = body[:body.index("\n}")]
    c = re.search(r"rcpf\(fmaf\(([0-9.]+)f, fabsf\(x\), 1\.f\)\)", body).group(1)
    first = re.search(r"float s = (-?[0-9.]+)f;", body).group(1)
    rest = re.findall(r"s = fmaf\(s, t, (-?[0-9.]+)f\);", body)
    assert len(rest) == 7
    return np.array([first] + rest, dtype=np.float32).astype(np.float64), float(np.float32(c))


def test_fit_over_its_range():
    s, c = _coefficients()
    a = np.concatenate([np.linspace(0, 40, 400001), np.geomspace(1e-9, 1, 20001)])
    t = 1 / (1 + c * a)
    exact = erfcx(a / np.sqrt(2)) / 2                                     # Q(a) exp(a^2 / 2)
    assert np.abs(t * np.polyval(s, t) / exact - 1).max() <= 4.5e-7


def test_half_at_zero():
    """P(0) = 1/2, in fp32 operation by operation as well: gelu's slope does not jump where x changes its sign."""
    s, _ = _coefficients()
    assert s.sum() == 0.5
    at = np.float32(s[0])
    for v in s[1:]:
        at = np.float32(float(at) + v)
    assert at == np.float32(0.5)
