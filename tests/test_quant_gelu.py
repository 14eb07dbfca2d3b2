"""The GELU of float32 outputs of the 8-bit linear layer (csrc/quant_linear.hip): its coefficients
are the degree-11 fit of paper_2407_02068_amd/gelu_fit.py, and the kernel's formula, step by step in
float32, meets the accuracy its comment states (host logic; no GPU)."""
import os
import re

import numpy as np
from scipy.special import erfc

from paper_2407_02068_amd import gelu_fit
from test_gelu_fit import gelu32

SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2407_02068_amd", "csrc", "quant_linear.hip")


def coefficients():
    body = open(SRC).read()
    body = body[body.index("__device__ inline float gelu_f32(float v)"):]
    body = body[:body.index("__builtin_amdgcn_exp2f")]
    vals = [float(v) for v in re.findall(r"(-?\d\.\d+e[-+]\d+)f", body)]
    return np.array(vals[::-1], dtype=np.float32)


def test_coefficients_are_the_fit():
    np.testing.assert_allclose(coefficients(), gelu_fit.fit(11), rtol=1e-8, atol=0)


def test_accuracy():
    """The kernel's steps in float32 against x Phi(x) in float64, each output within the bound of its own
    roundings.  e = 2^(f(a) - 1/2): a = |x| / sqrt 2 is off by two roundings (of the constant and of the
    product), 2^-23 a, which moves f by |f'(a)| a 2^-23; step k of the fused Horner scheme is off by half
    a unit of its value r_k, which reaches f times a^k; 2^d is off by ln 2 d relative.  To that come the
    fit's own error, the roundings of e and of a (2^-23), and the output's (2^-24)."""
    c = coefficients()
    x = np.linspace(-5.5, 40.0, 910001).astype(np.float32)
    x = x[x != 0]
    xd = x.astype(np.float64)
    ref = xd * 0.5 * erfc(-xd / np.sqrt(2.0))
    err = np.abs(gelu32(x, c).astype(np.float64) - ref)
    a = np.minimum(np.abs(xd) / np.sqrt(2.0), 4.0)
    f = c.astype(np.float64)
    fit = np.abs(np.exp2(np.polyval(f[::-1], a)) / erfc(a) - 1.0)
    slope = np.abs(np.polyval((f[1:] * np.arange(1, 12))[::-1], a)) * a * 2.0**-23
    horner, r = np.zeros_like(a), np.zeros_like(a) + f[-1]
    for k in range(10, -1, -1):
        r = r * a + (f[k] - 0.5 if k == 0 else f[k])
        horner += np.abs(r) * a**k * 2.0**-24
    rel = fit + np.log(2.0) * (slope + horner) * 1.01 + 2 * 2.0**-23  # of the term a e
    term = np.where(np.abs(xd) / np.sqrt(2.0) < 4.0, a * erfc(a) / np.sqrt(2.0), 0.0)
    cut = np.where(np.abs(xd) / np.sqrt(2.0) < 4.0, 0.0, np.abs(np.maximum(xd, 0) - ref))
    assert (err <= term * rel + np.abs(ref) * 2.0**-24 + cut).all()
    # what include/lpv.h states
    assert (err[x > 0] / ref[x > 0]).max() < 3e-7
    tail = x < 0
    assert (err[tail] / np.abs(ref[tail])).max() < 8e-6 and err[tail].max() < 1e-7


def test_special_values():
    g = gelu32(np.array([np.inf, -np.inf, 0.0], np.float32), coefficients())
    assert g[0] == np.inf and g[1] == 0.0 and g[2] == 0.0
