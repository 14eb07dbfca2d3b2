"""Tokens whose scale is near the largest float32 (rows that hold a type's lowest value) through
the 8-bit linear layer: a sum times the scale may pass the largest float32 where the output does not."""
import numpy as np
import pytest
import torch

from oracle import quant
from gpu_util import TORCH, f64, kernels
from test_gpu_quant_linear import Case, check, lpv

pytestmark = pytest.mark.gpu

# one size for each kernel
SIZES = [(33, 96, 512, 0, "few<%d, %s, 4, 4>"), (1, 256, 4096, 0, "few<%d, %s, 8, 4>"),
         (1000, 1600, 80, 16, "panel<%d, %s, 1, 4, 4>"), (1500, 8208, 336, 16, "panel<%d, %s, 2, 4, 4>"),
         (5000, 8208, 592, 16, "panel<%d, %s, 4, 4, 2>"), (2050, 8208, 2064, 16, "panel<%d, %s, 4, 8, 4>")]


def far_case(M, N, K, b, dtype):
    """Every third token's scale is 2^112 to 2^126 (float16: 2^118), the weight's scales small."""
    c = Case(M, N, K, dtype, b, b, 45)
    g = torch.Generator(device="cuda").manual_seed(M)
    e = torch.rand((M + 2) // 3, generator=g, device="cuda") * (6 if dtype == "f16" else 14)
    c.xs[::3] = torch.exp2(112 + e) * torch.where(torch.arange(e.numel(), device="cuda") % 2 == 0, 1.0, -1.0)
    c.ws *= 2.0 ** -63
    c.ws *= 2.0 ** -63 if dtype == "f16" else 1.0  # (some of them are subnormal)
    return c


@pytest.mark.parametrize("M,N,K,b,kernel", SIZES)
def test_every_kernel(M, N, K, b, kernel):
    for dtype, code in (("bf16", 2), ("f16", 1), ("f32", 0)):
        if dtype == "f32" and "4, 4, 2" in kernel:
            continue
        for gelu in (False, True):
            c = far_case(M, N, K, b, dtype)
            h, epi = c.pack(), "gelu" if gelu else None
            run = lambda i, xs: lpv().quant_linear(h, c.X[i], xs[i], c.bias, epi=epi)
            Y = run(slice(None), c.xs)
            assert kernels(lambda: run(slice(None), c.xs), args=True) == {"k_quant_" + kernel % (code, str(gelu).lower())}
            at = slice(0, 70)
            part = far_case(M, N, K, b, dtype)
            part.X, part.xs = c.X[at], c.xs[at]
            check(Y[at], part.want(gelu), dtype, gelu, "%s far" % (kernel % (code, gelu)))
            # a row's bits are its own: alone, and beside tokens of ordinary scales
            for i in {0, M // 2, M - 1}:
                assert torch.equal(run(slice(i, i + 1), c.xs)[0], Y[i]), i
            near = c.xs.clone()
            near[::3] = 0.25
            other = run(slice(None), near)
            rest = torch.arange(M, device="cuda") % 3 != 0
            assert torch.equal(Y[rest], other[rest])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [3, 3000])
def test_a_types_lowest_value_in_a_row(dtype, M):
    # -3.4e38 where a mask left nothing, into a layer that makes it smaller
    K, N = 512, 1040
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((M, K), generator=g, device="cuda").to(TORCH[dtype])
    x[1, 3] = torch.finfo(x.dtype).min
    x[M - 1] = torch.finfo(x.dtype).min
    w = torch.randn((N, K), generator=g, device="cuda") * 1e-4
    q, xs = lpv().quant_rows(x)
    wq, ws = lpv().quant_rows(w)
    ref = quant.linear(q[-3:].cpu().numpy(), f64(xs[-3:]), wq.cpu().numpy(), f64(ws))
    for epi in (None, "gelu"):
        Y = lpv().quant_linear(lpv().quant_pack(wq, ws), q, xs, dtype=x.dtype, epi=epi)
        assert torch.isfinite(Y).all()
        if epi is None:
            check(Y[-3:], ref, dtype, False, "lowest value")
            assert float(Y[M - 1].abs().max()) > 1e34


def test_scales_that_are_not_finite_and_weights_as_large():
    """What is infinite stays so, and a sum of 0 is 0 whatever the finite scales are."""
    c = Case(40, 96, 64, "f32", bias=False)
    c.X[5] = 0
    c.xs[5:9] = torch.tensor([3e38, 3e38, float("inf"), float("nan")], device="cuda")
    c.ws[:] = 3e38
    Y = lpv().quant_linear(c.pack(), c.X, c.xs, dtype=torch.float32)
    assert not Y[5].any()
    s = c.X[6:8].cpu().double() @ c.W.cpu().double().t()
    for row, total in zip(Y[6:8].cpu(), s):
        assert torch.equal(row[total != 0].double(), total[total != 0].sign() * float("inf"))
    assert not Y[6][s[0].cuda() == 0].any()
    assert Y[8].isnan().all()
