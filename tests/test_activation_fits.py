"""The polynomials of csrc/linear_epilogue.h, as the header holds them, against 64-bit functions."""
import math
import os
import re

import torch

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_23472_amd", "csrc", "linear_epilogue.h")


def _coefficients(name):
    """Of `float name = c0;` and the `name = fmaf(name, ., c);` that follow, highest power first."""
    text = open(HEADER).read()
    first = re.search(r"float %s = (-?[0-9.e-]+)f;" % name, text).group(1)
    return [float(c) for c in [first] + re.findall(r"%s = fmaf\(%s, \w, (-?[0-9.e-]+)f\);" % (name, name), text)]


def _horner(coefficients, at):
    v = torch.zeros_like(at)
    for c in coefficients:
        v = v * at + float(torch.tensor(c, dtype=torch.float32))
    return v


def test_erfc():
    x = torch.cat([torch.linspace(0, 12, 20001, dtype=torch.float64), torch.logspace(-8, 3, 2001, dtype=torch.float64)])
    t = 1 / (1 + 0.4 * x)
    q = _coefficients("q")
    assert len(q) == 9
    want = torch.special.erfcx(x)                        # exp(x^2) erfc(x)
    assert ((_horner(q, t) * t - want).abs() / want).max() < 1.45e-7


def test_phi_near_zero():
    z = torch.linspace(-math.sqrt(2), math.sqrt(2), 20001, dtype=torch.float64)
    r = _coefficients("r")
    assert len(r) == 7
    assert (z * _horner(r, z * z) - 0.5 * torch.erf(z / math.sqrt(2))).abs().max() < 2e-8
