"""Rows in 8-bit codes on the GPU (alone, and behind the residual's addition and a norm) against
the float64 oracle: the codes are equal, the scales within their one rounding."""
import numpy as np
import pytest
import torch

from oracle import quant
from gpu_util import TORCH, f64, say

pytestmark = pytest.mark.gpu

EPS = 1e-6


def lpv():
    from paper_2407_02068_amd import lpv as m
    m.lib()
    return m


def make(M, D, dtype, seed, wide=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x = n(M, D) * (torch.exp(n(D)) if wide else 1)
    return [t.to(TORCH[dtype]) for t in (x, n(M, D), 1 + 0.3 * n(D), 0.3 * n(D))]


def call(kind, x, y, g, b, eps=EPS, **kw):
    m = lpv()
    if kind == "rms":
        return m.add_rmsnorm_quant(x, y, g, eps, **kw)
    if kind == "layer":
        return m.add_layernorm_quant(x, y, g, b, eps, **kw)
    return m.quant_rows(x, y, **kw)


def want(kind, x, y, g, b, eps=EPS):
    s = f64(x) if y is None else f64(x) + f64(y)
    if kind == "rms":
        return quant.rms(s, f64(g), eps)
    if kind == "layer":
        return quant.layer(s, f64(g), f64(b), eps)
    return quant.codes(s)


def check(got, ref, what=""):
    """Equal codes: both sides are in float64 with errors under 2^-40 of a code, so that a value
    would have to lie that near a border to differ.  A scale: one rounding to float32, 2^-24
    relative (2^-150 below the normal numbers), and float64 errors before it."""
    q, scale = got[0].cpu().numpy().astype(np.int64), got[1].cpu().numpy().astype(np.float64)
    off = int((q != ref[0]).sum())
    nan = np.isnan(ref[1])
    assert (np.isnan(scale) == nan).all(), what
    err = np.abs(scale - ref[1])[~nan] - (2.0 ** -24 * (1 + 1e-6) * ref[1][~nan] + 2.0 ** -150)
    say("  %s: %d of %d codes differ, scales over their bound by %.3g" % (what, off, q.size, err.max(initial=-1)))
    assert off == 0, what
    assert (err <= 0).all(), what


def sum_of(x, y):
    return (x.float() + y.float()).to(x.dtype)  # (lpv_add_layernorm's: float32, one rounding)


# every kernel's sizes (rows of a wave, 256 and 1024 threads), their ends, odd lengths
SIZES = [(1, 1), (3, 2), (5, 7), (2, 8), (7, 16), (33, 63), (4, 64), (9, 511), (6, 512), (5, 513), (3, 520),
         (64, 768), (5, 1000), (2, 1023), (7, 1024), (2, 1025), (3, 1032), (4, 2048), (2, 2049), (3, 3000),
         (2, 4096), (2, 4100), (3, 5120), (1, 8192), (2, 8200), (1, 9001), (2, 16384), (1, 16392), (2, 20001),
         (1, 32768), (1, 32767)]


@pytest.mark.parametrize("M,D", SIZES)
@pytest.mark.parametrize("kind", ["plain", "rms", "layer"])
def test_sizes(kind, M, D):
    for i, dtype in enumerate(("bf16", "f16", "f32")):
        x, y, g, b = make(M, D, dtype, 17 * D + i)
        if kind == "layer" and D == 1:
            b = b + 1  # (a row of one value is beta alone: its codes are 127 or -127)
        S = torch.empty_like(x)
        got = call(kind, x, y, g, b, S=S)
        check(got, want(kind, x, y, g, b), "%s %s %d x %d" % (kind, dtype, M, D))
        assert torch.equal(S, sum_of(x, y))
        got = call(kind, x, None, g, b)
        check(got, want(kind, x, None, g, b), "%s %s %d x %d alone" % (kind, dtype, M, D))


@pytest.mark.parametrize("kind", ["plain", "rms", "layer"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_many_rows(kind, dtype):
    x, y, g, b = make(1777, 384, dtype, 5)
    S = torch.empty_like(x)
    check(call(kind, x, y, g, b, S=S), want(kind, x, y, g, b), "many")
    assert torch.equal(S, sum_of(x, y))


@pytest.mark.parametrize("kind", ["plain", "rms", "layer"])
@pytest.mark.parametrize("D,pad,first", [(40, 8, 0), (40, 3, 0), (40, 8, 1), (37, 3, 0), (768, 16, 0), (1500, 1, 3),
                                         (4096, 64, 0), (2056, 8, 4)])
def test_strides_and_what_lies_around(kind, D, pad, first):
    # inputs and outputs in the middle of wider rows, aligned and not; nothing else is written
    M, dtype = 11, "bf16"
    x, y, g, b = make(M, D, dtype, D + pad)
    W = D + pad + first
    at = slice(first, first + D)
    wide = {}
    for name, t in (("x", x), ("y", y)):
        wide[name] = torch.full((M + 2, W), float("nan"), dtype=x.dtype, device="cuda")
        wide[name][1:-1, at] = t
    S = torch.full((M + 2, W), 7.0, dtype=x.dtype, device="cuda")
    q = torch.full((M + 2, W), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((M + 2,), -5.0, device="cuda")
    keep_x = wide["x"].clone()
    view = lambda t: t[1:-1, at]
    got = call(kind, view(wide["x"]), view(wide["y"]), g, b, S=view(S), q=view(q), scale=scale[1:-1])
    check(got, want(kind, x, y, g, b), "strided")
    assert torch.equal(view(S), sum_of(x, y))
    for t, v in ((S, 7.0), (q, 99)):
        t[1:-1, at] = v
        assert (t == v).all()
    assert scale[0] == -5 and scale[-1] == -5
    assert torch.equal(wide["x"].nan_to_num(1e4), keep_x.nan_to_num(1e4))


@pytest.mark.parametrize("kind", ["plain", "rms", "layer"])
@pytest.mark.parametrize("D", [96, 777, 3000])
def test_the_sum_in_place_of_an_input(kind, D):
    for which in (0, 1):
        x, y, g, b = make(9, D, "f16", D)
        ref, S = want(kind, x, y, g, b), sum_of(x, y)
        t = (x, y)[which]
        check(call(kind, x, y, g, b, S=t), ref, "in place")
        assert torch.equal(t, S)


@pytest.mark.parametrize("kind", ["plain", "rms", "layer"])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 1100), ("f16", 5000), ("f16", 333)])
def test_rows_that_are_empty_huge_tiny_or_not_finite(kind, dtype, D):
    big = {"bf16": 3e38, "f16": 6e4, "f32": 3e38}[dtype]
    small = {"bf16": 1e-38, "f16": 6e-8, "f32": 1e-38}[dtype]
    x, _, g, b = make(9, D, dtype, 3, wide=False)
    x = x.float().clamp(-1, 1)
    x[0] = 0
    x[1] *= big
    x[2] *= small
    x[3, D // 2] = float("nan")
    x[4, D - 1] = float("inf")
    x[5, 0] = float("-inf")
    x[6] = 0
    x[6, D - 1] = small * 4
    x[7] = 1.5
    x = x.to(TORCH[dtype])
    if kind == "layer":
        b = torch.zeros_like(b)  # (a constant row is then zero, not its beta)
    check(call(kind, x, None, g, b), want(kind, x, None, g, b), "%s %s" % (kind, dtype))
    # without eps: a row of zeros is zero behind a root-mean-square norm, and has no layer norm
    if kind != "plain":
        check(call(kind, x, None, g, b, eps=0.0), want(kind, x, None, g, b, eps=0.0), "eps = 0")


def test_a_parameter_that_is_not_finite():
    x, y, g, b = make(5, 200, "bf16", 8)
    g[7] = float("inf")
    for kind in ("rms", "layer"):
        q, scale = call(kind, x, y, g, b)
        assert scale.isnan().all() and not q.any()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_quotients_halfway_between_two_codes(dtype):
    # a largest value of 127 * 2^k, and every half of a code: to the even neighbour, either sign
    h = torch.arange(-254, 255, device="cuda").float() / 2
    rows = torch.stack([h * f for f in (1.0, 0.25, 64.0, 2.0 ** -10)])
    if dtype == "bf16":
        rows = rows[:, 0::1]  # (509 halves up to 127: 8 bits each)
    x = rows.to(TORCH[dtype])
    assert torch.equal(x.float(), rows)
    q, scale = lpv().quant_rows(x)
    assert torch.equal(q.float(), torch.round(h).expand_as(q))
    ones = torch.ones(h.numel(), dtype=x.dtype, device="cuda")
    q, _ = lpv().add_rmsnorm_quant(x, None, ones, EPS)
    assert torch.equal(q.float(), torch.round(h).expand_as(q))
    # a largest value that is no power of two times 127: 3 u / m with m = 381 / 2 ...
    u = torch.tensor([[190.5, 0.75, 2.25, -3.75, 5.25, 1.5]], device="cuda").to(TORCH[dtype])
    check(lpv().quant_rows(u), quant.codes(f64(u)), "thirds")


def test_refusals_of_the_binding():
    m = lpv()
    x, y, g, b = make(4, 32, "bf16", 1)
    for bad in (lambda: m.quant_rows(x[0]), lambda: m.quant_rows(x.to(torch.float64)), lambda: m.quant_rows(x.cpu()),
                lambda: m.quant_rows(x, y.half()), lambda: m.quant_rows(x, y[:3]), lambda: m.quant_rows(x.t()),
                lambda: m.quant_rows(x, S=y.float()), lambda: m.quant_rows(x, q=torch.empty(4, 32, device="cuda")),
                lambda: m.quant_rows(x, scale=torch.empty(4, dtype=torch.float64, device="cuda")),
                lambda: m.quant_rows(x, scale=torch.empty(4)),
                lambda: m.add_rmsnorm_quant(x, y, g[:16], EPS), lambda: m.add_rmsnorm_quant(x, y, g.float(), EPS),
                lambda: m.add_rmsnorm_quant(x, y, g.cpu(), EPS), lambda: m.add_rmsnorm_quant(x, y, None, EPS),
                lambda: m.add_layernorm_quant(x, y, g, b[None], EPS)):
        with pytest.raises((ValueError, TypeError, AttributeError)):
            bad()
    with pytest.raises(m.LpvError, match="LPV_ERR_ALIAS"):
        m.quant_rows(x, q=x.view(torch.int8)[:, :32])
    with pytest.raises(m.LpvError, match="LPV_ERR_SHAPE"):
        m.quant_rows(torch.zeros(1, 32769, device="cuda"))
    q, scale = m.quant_rows(x[:0])
    assert q.shape == (0, 32) and scale.shape == (0,)


def test_another_stream_and_a_captured_graph():
    m = lpv()
    x, y, g, b = make(300, 768, "bf16", 2)
    ref = [t.clone() for t in m.add_layernorm_quant(x, y, g, b, EPS)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = m.add_layernorm_quant(x, y, g, b, EPS)
    q, scale = torch.empty_like(ref[0]), torch.empty_like(ref[1])
    m.add_layernorm_quant(x, y, g, b, EPS, q=q, scale=scale, stream=side)
    side.synchronize()
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    assert torch.equal(q, ref[0]) and torch.equal(scale, ref[1])
    S = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.add_rmsnorm_quant(x, y, g, EPS, S=S, q=q, scale=scale)
    for k in range(3):
        x.copy_(x.flip(0))
        want_q, want_s = m.add_rmsnorm_quant(x, y, g, EPS)
        q.zero_()
        scale.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, want_q) and torch.equal(scale, want_s) and torch.equal(S, sum_of(x, y)), k


@pytest.mark.parametrize("kind", ["plain", "rms", "layer"])
def test_a_stream_that_is_not_current_takes_its_outputs(kind):
    """New outputs come from the current stream's memory: a call on another one is refused without
    its outputs, one of them missing or both."""
    x, y, g, b = make(4, 64, "bf16", 3)
    side = torch.cuda.Stream()
    q, scale = torch.empty((4, 64), dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    for kw in ({}, {"q": q}, {"scale": scale}):
        with pytest.raises(ValueError, match="takes its outputs"):
            call(kind, x, y, g, b, stream=side, **kw)
    got = call(kind, x, y, g, b, stream=torch.cuda.current_stream())
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        again = call(kind, x, y, g, b, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
