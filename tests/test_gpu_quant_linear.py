"""The linear layer over 8-bit codes on the GPU against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import quant
from gpu_util import TORCH, f64, kernels, say

pytestmark = pytest.mark.gpu


def lpv():
    from paper_2407_02068_amd import lpv as m
    m.lib()
    return m


class Case:
    """Codes of every value, scales over some powers of two, and (block > 0) a random mask."""

    def __init__(self, M, N, K, dtype="bf16", b_r=0, b_c=0, drop=50, bias=True, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed + 7 * M + 11 * N + 13 * K)
        codes = lambda *s: torch.randint(-128, 128, s, generator=g, device="cuda").to(torch.int8)
        scales = lambda n: torch.exp2(4 * torch.randn(n, generator=g, device="cuda") - 10)
        self.dtype, self.M, self.N, self.K, self.b_r, self.b_c = dtype, M, N, K, b_r, b_c
        self.X, self.W, self.xs, self.ws = codes(M, K), codes(N, K), scales(M) * 2.0 ** -3, scales(N)
        # outputs of about 1, so that the bias counts
        self.ws *= 2.0 ** 20 / (6000 * K ** 0.5) * 2.0 ** -2
        self.bias = torch.randn(N, generator=g, device="cuda").to(TORCH[dtype]) if bias else None
        self.mask = None
        if b_c:
            r = torch.rand((N // b_r, K // b_c), generator=g, device="cuda") * 100
            self.mask = (r >= drop).to(torch.uint8)

    def pack(self):
        if self.mask is None:
            return lpv().quant_pack(self.W, self.ws)
        return lpv().quant_pack(self.W, self.ws, self.mask, self.b_r, self.b_c)

    def want(self, gelu=False):
        W = self.W.cpu().numpy()
        if self.mask is not None:
            W = quant.keep(W, self.mask.cpu().numpy(), self.b_r, self.b_c)
        return quant.linear(self.X.cpu().numpy(), f64(self.xs), W, f64(self.ws),
                            None if self.bias is None else f64(self.bias), gelu)


def check(Y, ref, dtype, gelu=False, what=""):
    """The sum is converted to float32, takes the token's scale, then the output's with the bias
    in one fused step: 2^-24 each, the first two relative to the product A (GELU's slope is
    at most 1.13; its own error is 5e-6 relative, and below 5e-8 |v| where it becomes max(v, 0)).
    A 16-bit output is rounded once more, by half a step (fp16: at least 2^-25)."""
    y, (r, A) = f64(Y), ref
    bound = 2.0 ** -24 * (2.01 * A + 1.01 * np.maximum(np.abs(r), 0 if not gelu else A + np.abs(r)))
    if gelu:
        bound = 1.13 * bound + 5e-6 * np.abs(r) + 5e-8 * A + 1e-37
    half = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 0.0}[dtype]
    bound = bound * (1 + half) + half * np.abs(r) + (2.0 ** -25 if dtype == "f16" else 1e-38)
    off = np.abs(y - r)
    big = np.abs(r) >= 65504 if dtype == "f16" else np.zeros(r.shape, bool)
    worst = float((off / bound)[~big].max(initial=0.0))
    say("  %s: %.3g of its bound" % (what, worst))
    assert np.isfinite(y[~big]).all() and worst <= 1.0, what


DENSE = [(1, 16, 16), (1, 32, 48), (2, 48, 32), (31, 64, 64), (32, 80, 496), (33, 96, 512), (63, 512, 528),
         (64, 528, 1024), (65, 560, 1040), (127, 64, 2064), (128, 1040, 768), (129, 1024, 80), (197, 2304, 768),
         (1, 4096, 4096), (5, 176, 8208), (257, 96, 1600), (500, 1536, 384), (1000, 272, 304),
         (1100, 8208, 80), (2050, 8208, 80), (8300, 2064, 560), (600, 8208, 1072)]


@pytest.mark.parametrize("M,N,K", DENSE)
def test_dense(M, N, K):
    for dtype, gelu in (("bf16", False), ("f16", True), ("f32", False)):
        c = Case(M, N, K, dtype)
        Y = lpv().quant_linear(c.pack(), c.X, c.xs, c.bias, epi="gelu" if gelu else None)
        assert Y.dtype == TORCH[dtype]
        check(Y, c.want(gelu), dtype, gelu, "dense %d x %d x %d %s" % (M, N, K, dtype))


BLOCKS = [(1, 64, 64, 16, 16, 50), (7, 64, 64, 64, 64, 50), (33, 96, 48, 16, 16, 60), (64, 128, 512, 32, 32, 50),
          (65, 112, 560, 16, 16, 90), (197, 2304, 768, 32, 32, 50), (130, 576, 1088, 64, 64, 80),
          (300, 1536, 384, 16, 16, 75), (1, 1024, 2048, 32, 64, 95), (129, 544, 1056, 32, 16, 30),
          (77, 640, 1600, 64, 32, 99), (513, 192, 4096, 16, 64, 40), (260, 320, 512, 64, 16, 0),
         (2050, 8208, 112, 16, 16, 70), (1030, 8192, 1088, 64, 32, 60), (520, 8224, 1072, 32, 16, 85),
         (17000, 1088, 576, 64, 64, 30)]


@pytest.mark.parametrize("M,N,K,b_r,b_c,drop", BLOCKS)
def test_blocks(M, N, K, b_r, b_c, drop):
    for dtype, gelu in (("bf16", True), ("f16", False), ("f32", False)):
        c = Case(M, N, K, dtype, b_r, b_c, drop)
        h = c.pack()
        assert h.info["nnzb"] == int(c.mask.sum()) and (h.info["R"], h.info["C"]) == tuple(c.mask.shape)
        Y = lpv().quant_linear(h, c.X, c.xs, c.bias, epi="gelu" if gelu else None)
        check(Y, c.want(gelu), dtype, gelu, "%d x %d x %d, %d x %d blocks %s" % (M, N, K, b_r, b_c, dtype))


@pytest.mark.parametrize("M,N,K,b,kernel", [
    (33, 96, 512, 0, "few<%d, %s, 4, 4>"), (1, 256, 4096, 0, "few<%d, %s, 8, 4>"),
    (1000, 1600, 80, 16, "panel<%d, %s, 1, 4, 4>"), (1500, 8208, 336, 16, "panel<%d, %s, 2, 4, 4>"),
    (5000, 8208, 592, 16, "panel<%d, %s, 4, 4, 2>"), (2050, 8208, 2064, 16, "panel<%d, %s, 4, 8, 4>")])
def test_every_kernel(M, N, K, b, kernel):
    # the size that reaches it, in every type, with and without GELU: the ends against the oracle, the
    # rows between against the same rows in a call of their own
    for dtype, code in (("bf16", 2), ("f16", 1), ("f32", 0)):
        if dtype == "f32" and "4, 4, 2" in kernel:
            continue
        for gelu in (False, True):
            c = Case(M, N, K, dtype, b, b, 45)
            h = c.pack()
            epi = "gelu" if gelu else None
            Y = lpv().quant_linear(h, c.X, c.xs, c.bias, epi=epi)
            assert kernels(lambda: lpv().quant_linear(h, c.X, c.xs, c.bias, epi=epi), args=True) == {
                "k_quant_" + kernel % (code, str(gelu).lower())}
            for at in ([slice(0, 70), slice(max(0, M - 70), M)] if M > 140 else [slice(0, M)]):
                part = Case(M, N, K, dtype, b, b, 45)
                part.X, part.xs = c.X[at], c.xs[at]
                check(Y[at], part.want(gelu), dtype, gelu, "%s rows %s" % (kernel % (code, gelu), at))
            if M > 64:
                for i in range(0, M - 32, max(32, (M // 8) & ~15)):
                    few = lpv().quant_linear(h, c.X[i:i + 32], c.xs[i:i + 32], c.bias, epi=epi)
                    assert torch.equal(Y[i:i + 32], few), i


@pytest.mark.parametrize("M", [1, 40, 300, 5000])
@pytest.mark.parametrize("which", ["none", "one", "last", "row", "column"])
def test_masks_that_leave_rows_columns_or_everything_empty(M, which):
    c = Case(M, 1120, 1600, "f32", 32, 32)
    c.mask.zero_()
    if which == "one":
        c.mask[3, 7] = 1
    if which == "last":
        c.mask[-1, -1] = 255  # (nonzero keeps)
    if which == "row":
        c.mask[17] = 1
    if which == "column":
        c.mask[:, 20] = 1
    h = c.pack()
    Y = lpv().quant_linear(h, c.X, c.xs, c.bias)
    check(Y, c.want(), "f32", False, which)
    if which == "none":
        assert torch.equal(Y, c.bias.expand_as(Y))
        assert not lpv().quant_linear(h, c.X, c.xs, dtype=torch.float32).any()


def test_a_dense_mask_and_no_mask_give_the_same_bits():
    c = Case(150, 144, 1040, "bf16")
    a = lpv().quant_linear(c.pack(), c.X, c.xs, c.bias)
    ones = torch.ones((9, 65), dtype=torch.uint8, device="cuda")
    b = lpv().quant_linear(lpv().quant_pack(c.W, c.ws, ones, 16, 16), c.X, c.xs, c.bias)
    assert torch.equal(a, b)


def test_the_weight_comes_back_through_unit_tokens():
    # X = 100 I: column k of the weight; every code and every place of a tile
    c = Case(1040, 560, 1040, "f32", 16, 16, 40, bias=False)
    c.X = (100 * torch.eye(1040, device="cuda")).to(torch.int8)
    ones = torch.ones(1040, device="cuda")
    h = lpv().quant_pack(c.W, ones[:560].contiguous(), c.mask, 16, 16)
    Y = lpv().quant_linear(h, c.X, ones, dtype=torch.float32)
    W = quant.keep(c.W.cpu().numpy(), c.mask.cpu().numpy(), 16, 16)
    assert np.array_equal(Y.cpu().numpy().T, 100.0 * W)


@pytest.mark.parametrize("M,K", [(1, 65536), (40, 65536), (300, 65536), (5000, 8192)])
def test_the_largest_sums(M, K):
    # every product 2^14: sums of 2^30, and alternating ones that cancel
    X = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    W = torch.full((64, K), -128, dtype=torch.int8, device="cuda")
    W[1, ::2] = 127
    one = torch.ones(max(M, 64), device="cuda")
    h = lpv().quant_pack(W, one[:64])
    Y = lpv().quant_linear(h, X, one[:M], dtype=torch.float32)
    assert (Y[:, 0] == float(K * 2 ** 14)).all() and (Y[:, 1] == float(K // 2 * 128)).all()
    assert (Y[:, 2:] == float(K * 2 ** 14)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K,b", [(3, 48, 64, 0), (70, 80, 528, 16), (131, 1056, 544, 32), (700, 144, 1024, 0)])
def test_strides_and_what_lies_around(M, N, K, b, dtype):
    c = Case(M, N, K, dtype, b, b)
    X = torch.full((M + 2, K + 48), 77, dtype=torch.int8, device="cuda")
    X[1:-1, 16:16 + K] = c.X
    W = torch.full((N + 2, K + 32), -77, dtype=torch.int8, device="cuda")
    W[1:-1, 16:16 + K] = c.W
    Y = torch.full((M + 2, N + 16), 5.0, dtype=TORCH[dtype], device="cuda")
    xs = torch.full((M + 3,), float("nan"), device="cuda")
    xs[3:] = c.xs  # (12 bytes off: 4-byte alignment)
    ref = c.want()
    c.W = W[1:-1, 16:16 + K]
    lpv().quant_linear(c.pack(), X[1:-1, 16:16 + K], xs[3:], c.bias, Y=Y[1:-1, 8:8 + N])
    check(Y[1:-1, 8:8 + N], ref, dtype, False, "strided")
    Y[1:-1, 8:8 + N] = 5
    assert (Y == 5).all()


@pytest.mark.parametrize("M,N,K,b", [(1, 64, 256, 0), (64, 544, 768, 32), (1000, 1040, 1040, 0), (5000, 528, 1040, 16)])
def test_a_rows_bits_depend_on_no_other_row(M, N, K, b):
    c = Case(M, N, K, "bf16", b, b)
    h = c.pack()
    whole = lpv().quant_linear(h, c.X, c.xs, c.bias, epi="gelu")
    assert torch.equal(whole, lpv().quant_linear(h, c.X, c.xs, c.bias, epi="gelu"))
    for at in {0, M // 3, M - 1}:
        one = lpv().quant_linear(h, c.X[at:at + 1], c.xs[at:at + 1], c.bias, epi="gelu")
        assert torch.equal(one[0], whole[at]), at
    # a scale that is not finite is its row's
    xs = c.xs.clone()
    xs[M // 2] = float("nan")
    got = lpv().quant_linear(h, c.X, xs, c.bias, epi="gelu")
    assert got[M // 2].isnan().all()
    rest = torch.arange(M, device="cuda") != M // 2
    assert torch.equal(got[rest], whole[rest])


def test_many_rows_past_32_bit_offsets():
    # outputs of over 2^32 bytes: the last rows are as right as the first
    M, N, K = 140000, 16384, 32
    c = Case(64, N, K, "bf16")
    h = c.pack()
    part = lpv().quant_linear(h, c.X, c.xs, c.bias)
    X, xs = c.X.repeat(M // 64 + 1, 1)[:M], c.xs.repeat(M // 64 + 1)[:M]
    Y = lpv().quant_linear(h, X, xs, c.bias)
    for at in range(0, M - 64, 64 * 397):
        assert torch.equal(Y[at:at + 64], part), at
    assert torch.equal(Y[M - M % 64:], part[:M % 64])


def test_the_largest_weight():
    # 2^22 tiles, 4 GiB: tokens of one column each find theirs at either end
    n = 65536
    g = torch.Generator(device="cuda").manual_seed(3)
    W = torch.randint(-128, 128, (n, n), generator=g, device="cuda", dtype=torch.int8)
    ws, xs = torch.rand(n, generator=g, device="cuda"), torch.ones(300, device="cuda")
    h = lpv().quant_pack(W, ws)
    ks = torch.arange(300, device="cuda") * 219  # 0 ... 65481
    ks[-1] = n - 1
    X = torch.zeros((300, n), dtype=torch.int8, device="cuda")
    X[torch.arange(300, device="cuda"), ks] = 1
    for M in (3, 300):
        Y = lpv().quant_linear(h, X[-M:], xs[:M], dtype=torch.float32)
        assert torch.equal(Y, W[:, ks[-M:]].t().float() * ws), M


def test_streams_graph_and_two_weights():
    m = lpv()
    a, b = Case(333, 528, 768, "bf16", 16, 32), Case(333, 768, 528, "f16")
    ha, hb = a.pack(), b.pack()
    ra, rb = m.quant_linear(ha, a.X, a.xs, a.bias), m.quant_linear(hb, b.X, b.xs, b.bias)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    Y = torch.zeros_like(ra)
    torch.cuda.synchronize()
    m.quant_linear(ha, a.X, a.xs, a.bias, Y=Y, stream=side)
    with torch.cuda.stream(side):
        got = m.quant_linear(hb, b.X, b.xs, b.bias)
    again = m.quant_linear(ha, a.X, a.xs, a.bias)  # (beside it, on the first stream)
    torch.cuda.synchronize()
    assert torch.equal(Y, ra) and torch.equal(got, rb) and torch.equal(again, ra)
    Ya, Yb = torch.empty_like(ra), torch.empty_like(rb)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.quant_linear(ha, a.X, a.xs, a.bias, Y=Ya)
        m.quant_linear(hb, b.X, b.xs, b.bias, Y=Yb)
    for k in range(3):
        a.X.copy_(a.X.roll(1, 0))
        ra, rb = m.quant_linear(ha, a.X, a.xs, a.bias), m.quant_linear(hb, b.X, b.xs, b.bias)
        Ya.zero_()
        Yb.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Ya, ra) and torch.equal(Yb, rb), k


def test_refusals_of_the_binding():
    m = lpv()
    c = Case(4, 64, 96, "bf16", 32, 32)
    h = c.pack()
    for bad in (lambda: m.quant_linear(h, c.X[:, :64], c.xs), lambda: m.quant_linear(h, c.X.float(), c.xs),
                lambda: m.quant_linear(h, c.X, c.xs[:3]), lambda: m.quant_linear(h, c.X, c.xs.double()),
                lambda: m.quant_linear(h, c.X, None), lambda: m.quant_linear(h, c.X.cpu(), c.xs),
                lambda: m.quant_linear(h, c.X, c.xs.cpu()), lambda: m.quant_linear(h, c.X, c.xs, c.bias.half(), dtype=torch.bfloat16),
                lambda: m.quant_linear(h, c.X, c.xs, c.bias[:32]), lambda: m.quant_linear(h, c.X, c.xs, dtype=torch.int8),
                lambda: m.quant_linear(h, c.X, c.xs, Y=torch.empty(4, 63, device="cuda")),
                lambda: m.quant_linear(h, c.X, c.xs, Y=torch.empty(4, 64, device="cuda"), dtype=torch.float16),
                lambda: m.quant_linear(h, c.X, c.xs, epi="relu"),
                lambda: m.quant_pack(c.W.float(), c.ws), lambda: m.quant_pack(c.W, c.ws[:5]), lambda: m.quant_pack(c.W.cpu(), c.ws),
                lambda: m.quant_pack(c.W, c.ws, c.mask[:1], 32, 32), lambda: m.quant_pack(c.W, c.ws, c.mask.bool(), 32, 32)):
        with pytest.raises((ValueError, TypeError, KeyError)):
            bad()
    other = m.bsr_pack(torch.zeros((64, 96), dtype=torch.bfloat16, device="cuda"), c.mask, 32, 32)
    for bad in (other, None, h.handle):  # (a handle of another kind is no weight in 8-bit codes)
        with pytest.raises(ValueError):
            m.quant_linear(bad, c.X, c.xs)
    with pytest.raises(m.LpvError, match="LPV_ERR_BLOCK"):
        m.quant_pack(c.W, c.ws, torch.ones((8, 12), dtype=torch.uint8, device="cuda"), 8, 8)
    with pytest.raises(m.LpvError, match="LPV_ERR_SHAPE"):
        m.quant_pack(c.W[:, :88], c.ws)
    Y = m.quant_linear(h, c.X[:0], c.xs[:0])
    assert Y.shape == (0, 64) and Y.dtype == torch.bfloat16
    h.close()
    with pytest.raises(m.LpvError, match="LPV_ERR_INVALID_ARG"):
        m.quant_linear(h, c.X, c.xs)
    h.close()


def test_a_stream_that_is_not_current_takes_its_output():
    m = lpv()
    c = Case(5, 64, 96)
    h = c.pack()
    side = torch.cuda.Stream()
    with pytest.raises(ValueError, match="takes its outputs"):
        m.quant_linear(h, c.X, c.xs, c.bias, stream=side)
    assert torch.equal(m.quant_linear(h, c.X, c.xs, c.bias, stream=torch.cuda.current_stream()),
                       m.quant_linear(h, c.X, c.xs, c.bias))
