"""Codes of values next to the border of two codes on the GPU: those of the exact quotient of the row's
float64 values, in rational arithmetic.  A sum of two float32 or bfloat16 values, or a product with
gamma, can lie past a border by far less than an element of its own type can."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from gpu_util import TORCH, f64, say

pytestmark = pytest.mark.gpu


def lpv():
    from paper_2407_02068_amd import lpv as m
    m.lib()
    return m


def exact_codes(rows):
    """rint(127 u / max|u|) of rows of Fractions, ties to even (Python's round of a Fraction)."""
    tops = [max(abs(v) for v in row) for row in rows]
    return [[round(127 * u / m) for u in row] for row, m in zip(rows, tops)]


def fractions(x, y=None):
    """The float64 values of x, or of x + y."""
    return [[Fraction(v) for v in row] for row in (f64(x) if y is None else f64(x) + f64(y)).tolist()]


def check(q, rows, what):
    want = np.array(exact_codes(rows))
    off = int((q.cpu().numpy() != want).sum())
    say("  %s: %d of %d codes differ" % (what, off, want.size))
    assert off == 0, what


def near_ties(M, D, dtype, seed, far=52):
    """x and y whose sums are 127 2^a at one place of a row and (k + 1/2) 2^a (1 or -1) +- 2^(a - e), or
    no difference at all, at most of the others.  (A few with the largest e and k need more than
    float64's 53 bits: their values are the rounded sums.)"""
    r = np.random.default_rng(seed)
    # (float16 holds 2^-24 to 2^15: there e = 24 + a)
    a = np.full((M, 1), 6) if dtype == "f16" else r.integers(-12, 13, (M, 1))
    e = np.full((M, D), 30) if dtype == "f16" else r.integers(20, far, (M, D))
    x = (r.integers(0, 127, (M, D)) + 0.5) * np.exp2(a) * r.choice([-1, 1], (M, D))
    y = np.exp2((a - e).astype(np.float64)) * r.choice([-1, 0, 1], (M, D))
    top = r.integers(0, D, M)
    x[np.arange(M), top] = 127 * np.exp2(a[:, 0]) * r.choice([-1, 1], M)
    y[np.arange(M), top] = 0
    put = lambda v: torch.from_numpy(v).to("cuda", TORCH[dtype])
    xd, yd = put(x), put(y)
    assert np.array_equal(f64(xd), x) and np.array_equal(f64(yd), y)
    return xd, yd


def test_three_values():
    x = torch.tensor([[127.0, 0.5, 2.5]], device="cuda")
    y = torch.tensor([[0.0, 2.0 ** -42, 2.0 ** -42]], device="cuda")
    assert lpv().quant_rows(x, y)[0].tolist() == [[127, 1, 3]]
    assert lpv().quant_rows(x, -y)[0].tolist() == [[127, 0, 2]]
    assert lpv().quant_rows(-x, -y)[0].tolist() == [[-127, -1, -3]]
    assert lpv().quant_rows(x)[0].tolist() == [[127, 0, 2]]


# a row of a wave, of 256 and of 1024 threads; by one load and element by element
SIZES = [(40, 3), (9, 200), (7, 255), (5, 768), (4, 1000), (3, 1023), (3, 2048), (3, 2050), (2, 4096), (2, 4099),
         (1, 8192), (1, 12288), (1, 12289), (1, 32768), (1, 20001)]


@pytest.mark.parametrize("M,D", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_sums_past_a_tie(M, D, dtype):
    x, y = near_ties(M, D, dtype, 3 * D)
    rows = fractions(x, y)
    S = torch.empty_like(x)
    q, scale = lpv().quant_rows(x, y, S=S)
    check(q, rows, "sums %s %d x %d" % (dtype, M, D))
    assert torch.equal(S, (x.float() + y.float()).to(x.dtype))
    # behind a root-mean-square norm with gamma of one: the same codes; of -2: turned
    one = torch.ones(D, dtype=x.dtype, device="cuda")
    assert torch.equal(lpv().add_rmsnorm_quant(x, y, one, 1e-6)[0], q)
    assert torch.equal(lpv().add_rmsnorm_quant(x, y, -2 * one, 1e-6)[0], -q)
    # the scale: one rounding to float32 behind the float64 ones
    want = np.array([max(abs(v) for v in row) / 127 for row in rows], dtype=np.float64)
    assert (np.abs(scale.cpu().numpy() - want) <= 2.0 ** -24 * (1 + 1e-6) * want).all()


def products_near(target, lo, most):
    """Whole numbers a, b < 2^24 with a b within 2^-43 of target (relative) and not it, `most` of them
    on either side."""
    a = np.arange(lo, 2 * lo, dtype=np.int64)
    b = np.rint(target / a).astype(np.int64)
    d = a * b - target
    ok = (b < 1 << 24) & (d != 0) & (np.abs(d) <= target * 2.0 ** -43)
    low, high = np.flatnonzero(ok & (d < 0))[:most], np.flatnonzero(ok & (d > 0))[:most]
    at = np.concatenate([low, high])
    return a[at], b[at]


def test_products_past_a_tie():
    # s gamma = 254 2^39 at the row's largest place, (2 k + 1) 2^39 +- a little at the others
    s, g = [127 * 2.0 ** 17], [2.0 ** 23]
    for k in (0, 1, 2, 7, 40, 63, 99, 126):
        a, b = products_near((2 * k + 1) << 39, 1 << 22, 4)
        s += a.tolist()
        g += b.tolist()
    assert len(s) == 22  # (on both sides, of ties that are even below and above)
    x = torch.tensor([s, [-v for v in s]], dtype=torch.float32, device="cuda")
    gamma = torch.tensor(g, dtype=torch.float32, device="cuda")
    assert x[0].tolist() == s and gamma.tolist() == g
    rows = [[u * v for u, v in zip(row, fractions(gamma[None])[0])] for row in fractions(x)]
    check(lpv().add_rmsnorm_quant(x, None, gamma, 1e-6)[0], rows, "products")
    wide = torch.zeros((2, 3000), device="cuda")
    wide[:, 100:100 + len(s)] = x
    wide_gamma = torch.ones(3000, device="cuda")
    wide_gamma[100:100 + len(s)] = gamma
    q, _ = lpv().add_rmsnorm_quant(wide, None, wide_gamma, 1e-6)
    check(q[:, 100:100 + len(s)], rows, "products among 3000")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_random_sums_are_the_exact_quotients(dtype):
    # values of few bits: ties and everything around them
    g = torch.Generator(device="cuda").manual_seed(11)
    whole = lambda n: torch.randint(-n, n + 1, (60, 96), generator=g, device="cuda").to(TORCH[dtype])
    x, y = whole(250), whole(3) / 4
    rows = fractions(x, y)
    check(lpv().quant_rows(x, y)[0], rows, dtype)
    check(lpv().quant_rows(x)[0], fractions(x), dtype + " alone")
