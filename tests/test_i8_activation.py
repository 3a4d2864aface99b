"""GELU of the 8-bit products' bf16 results (csrc/pa_i8.hpp) on the CPU: its
coefficients, read from the source, evaluated in fp32 with fused multiply-adds
against 64 bits, to the errors that the source states."""
import math
import os
import re

import numpy as np
import pytest

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                   "paper_2502_02414_amd", "csrc", "pa_i8.hpp")


def _gelu(x):
    with open(SRC) as f:
        body = re.search(r"float gelu_for\(float x\) \{(.*?)\} else \{", f.read(), re.S).group(1)
    top = np.float32(re.search(r"minimum\(fabsf\(x\), ([\d.]+)f\)", body).group(1))
    c = [re.search(r"float p = ([-\d.e]+)f;", body).group(1)]
    c += re.findall(r"fmaf\(p, z, ([-\d.e]+)f\)", body)
    z = np.minimum(np.abs(x), top)
    p = np.full_like(z, np.float32(c[0]))
    for k in c[1:]:  # (the product of two fp32 values is exact in 64 bits)
        p = (p.astype(np.float64) * z + np.float64(np.float32(k))).astype(np.float32)
    q = np.exp2(p.astype(np.float64)).astype(np.float32)
    return (np.maximum(x, 0).astype(np.float64) - z.astype(np.float64) * q).astype(np.float32)


def _exact(x):
    return x.astype(np.float64) * 0.5 * np.array([math.erfc(-t / math.sqrt(2)) for t in
                                                  x.astype(np.float64)])


@pytest.mark.parametrize("lo,hi,bar", [(-3, 0, 1.8e-5), (-4, -3, 3.6e-5), (-6, -4, 1.1e-4),
                                       (-9, -6, 3.8e-4), (0, 20, 1.8e-5)])
def test_relative_error(lo, hi, bar):
    x = np.linspace(lo, hi, 20001).astype(np.float32)
    x = x[x != 0]
    assert np.max(np.abs(_gelu(x) / _exact(x) - 1)) <= 1.05 * bar


def test_behind_the_last_digits():
    x = np.linspace(-40, -9, 20001).astype(np.float32)
    assert np.max(np.abs(_gelu(x) - _exact(x))) <= 1.1e-18
