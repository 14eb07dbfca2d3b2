"""GPU parity of attention with a learned relative position bias, forward and gradients,
against the float64 oracle.

The tolerances are bounds on each element, made of the roundings that the kernels do: u is
half a step of the element type (2^-8 bf16, 2^-11 fp16).  A weight P_ij is off by u P_ij
(and by half the smallest step of fp16, 2^-25) for the products, and relative to its value
by f for the float32 arithmetic behind it; an output is rounded once more.  f covers the
score's error, at most (hd + 2) 2^-24 times the sum of its terms' magnitudes, taken twice
(in the score and in the row's sum), and 2^-20 for exp2, the sums and the division.  D is
formed from the rounded outputs, so it is off by sum_d |dout| E_out (and by 2^-17 of its
terms), which dS_ij takes P_ij times; dS is rounded by u |dS| for the products."""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from gpu_util import dev, f64, kernels, say
from oracle import finetune as ft
from paper_2407_02068_amd import lpv

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"bf16": 0.0, "f16": 2.0 ** -25}
LOWEST = {"bf16": -3.3895313892515355e38, "f16": -65504.0}


def window_index(s, extra=False):
    i = np.arange(s)
    y, x = np.repeat(i, s), np.tile(i, s)
    idx = (y[:, None] - y[None, :] + s - 1) * (2 * s - 1) + x[:, None] - x[None, :] + s - 1
    n = (2 * s - 1) ** 2
    if not extra:
        return idx.astype(np.int32), n
    full = np.empty((s * s + 1, s * s + 1), np.int32)
    full[1:, 1:] = idx
    full[0, :], full[:, 0], full[0, 0] = n, n + 1, n + 2
    return full, n + 3


def line_index(T, n=32):
    d = np.arange(T)[None, :] - np.arange(T)[:, None]
    return np.clip(d + n // 2, 0, n - 1).astype(np.int32), n


def gen(seed, shape, dtype, std=1.0):
    a = wl.quantize(wl.rng(seed, 0, 50).normal(0, std, shape).astype(np.float32), dtype)
    return a, oracle.decode(a, dtype).reshape(shape)


class Case:
    """Inputs on the device and as float64, and the float64 results."""

    def __init__(self, idx, n_buckets, n_seq, H, hd, dtype, region=None, seed=120, q_std=1.0,
                 edit=None):
        self.idx, self.n_seq, self.H, self.hd, self.dtype, self.region = idx, n_seq, H, hd, dtype, region
        self.T = T = idx.shape[0]
        M = n_seq * T
        q, self.x = gen(seed, (M, 3 * H * hd), dtype, q_std)
        t, self.t = gen(seed + 1, (n_buckets, H), dtype, 0.5)
        g, self.g = gen(seed + 2, (M, H * hd), dtype)
        self.qkv, self.table, self.dout = dev(q, dtype), dev(t, dtype), dev(g, dtype)
        if edit:
            edit(self)
        self.rp = lpv.relpos(torch.from_numpy(idx).cuda(), n_buckets)
        self.reg = None if region is None else torch.from_numpy(region.astype(np.int32)).cuda()

    def forward(self, **kw):
        lse = torch.full((self.n_seq, self.H, self.T), 7.0, dtype=torch.float32, device="cuda")
        out = lpv.relpos_attention(self.rp, self.table, self.qkv, self.n_seq, self.H,
                                   region=self.reg, lse=lse, hd=self.hd, **kw)
        return out, lse

    def grad(self, out, lse, **kw):
        return lpv.relpos_attention_grad(self.rp, self.table, self.qkv, out, lse, self.dout,
                                         self.n_seq, self.H, region=self.reg, hd=self.hd, **kw)

    def check(self, out, lse, dqkv=None, dtable=None):
        c, dt, hd, H, n, T = self, self.dtype, self.hd, self.H, self.n_seq, self.T
        u, tiny = U[dt], TINY[dt]
        r = ft.relpos_attention(c.x, c.t, c.idx, n, H, hd, region=c.region, dout=c.g,
                                lowest=LOWEST[dt])
        heads = lambda a: a.reshape(n, T, H, hd).transpose(0, 2, 1, 3)
        rows = lambda a: a.transpose(0, 2, 1, 3).reshape(n * T, H * hd)
        ds_abs = (hd + 2) * 2.0 ** -24 * r["abs_s"]  # error of a row's scores, n x H x T
        f = 2 * ds_abs + 2.0 ** -20
        x = np.nan_to_num(c.x, posinf=0.0, neginf=0.0).reshape(n, T, 3, H, hd)
        q, k, v = (np.abs(x[:, :, i]).transpose(0, 2, 1, 3) for i in range(3))
        g = np.abs(heads(np.nan_to_num(c.g, posinf=0.0, neginf=0.0)))  # (padding: not used)
        pv = heads(r["abs_pv"])
        e_out = (u + f[..., None] + T * 2.0 ** -24) * pv + u * np.abs(heads(r["out"])) \
            + tiny * (v.sum(2, keepdims=True) + 1)
        self.within(f64(out), r["out"], rows(e_out), "out")
        got, want = f64(lse), r["lse"]
        empty = want == -np.inf
        assert np.array_equal(got == -np.inf, empty)
        assert np.all(np.abs(got[~empty] - want[~empty]) <=
                      (ds_abs + 2.0 ** -21 * (2 + np.abs(np.where(empty, 0, want))))[~empty])
        if dqkv is None:
            return
        P, dP, D, B = r["P"], r["dP"], r["D"], r["abs_dP"]
        dS = P * (dP - D[..., None])
        # (e_out takes the output's own rounding too, which the kernel's D sees)
        e_D = (g * (1.02 * e_out + 2.0 ** -17 * np.abs(heads(r["out"])))).sum(3)
        f_P = f[..., None] + 2.0 ** -22 * (1 + np.abs(np.where(empty, 0, want)))[..., None]
        e_dS = P * (e_D[..., None] + f_P * (np.abs(dP) + np.abs(D)[..., None]) + hd * 2.0 ** -24 * B)
        e_dSr = 1.02 * e_dS + u * np.abs(dS) + tiny
        acc = (T + 8) * 2.0 ** -24
        sh = 1 / np.sqrt(hd)
        T_ = lambda a: a.transpose(0, 1, 3, 2)
        want = r["dqkv"].reshape(n, T, 3, H, hd).transpose(2, 0, 3, 1, 4)
        e = [sh * ((e_dSr + acc * np.abs(dS)) @ k), sh * (T_(e_dSr + acc * np.abs(dS)) @ q),
             T_(P * (u + f_P + acc) + tiny) @ g]
        got = f64(dqkv).reshape(n, T, 3, H, hd).transpose(2, 0, 3, 1, 4)
        for i, name in enumerate(("dQ", "dK", "dV")):
            self.within(got[i], want[i], 1.02 * e[i] + u * np.abs(want[i]) + tiny, name)
        e_t = np.zeros(c.t.shape)
        pairs = (e_dS + (n * T + 8) * 2.0 ** -24 * np.abs(dS)).sum(0)
        ok = c.idx >= 0
        for h in range(H):
            np.add.at(e_t[:, h], c.idx[ok], pairs[h][ok])
        self.within(f64(dtable), r["dtable"], 1.02 * e_t + u * np.abs(r["dtable"]) + tiny, "dtable")

    @staticmethod
    def within(got, want, bound, what):
        assert np.isfinite(got).all(), what + " is not finite"
        bound = bound + 1e-30
        worst = float((np.abs(got - want) / bound).max()) if got.size else 0.0
        say("  %s: at most %.2f of its bound (mean bound %.1e, mean value %.1e)"
            % (what, worst, bound.mean() if got.size else 0, np.abs(want).mean() if got.size else 0))
        assert worst <= 1.0, "%s: %.3g times its bound" % (what, worst)

    def run(self):
        out, lse = self.forward()
        dqkv, dtable = self.grad(out, lse)
        torch.cuda.synchronize()
        self.check(out, lse, dqkv, dtable)
        return out, lse, dqkv, dtable


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,n_seq,H,hd", [
    (1, 1, 1, 32), (1, 70, 3, 64), (2, 5, 2, 32), (31, 3, 2, 64), (32, 3, 1, 32), (33, 2, 3, 32),
    (63, 3, 2, 64), (64, 2, 2, 32), (65, 2, 1, 64), (96, 2, 2, 32), (127, 1, 2, 64),
    (128, 2, 1, 32), (129, 2, 1, 64), (161, 1, 2, 32), (223, 2, 1, 64), (224, 1, 2, 32),
    (225, 1, 2, 32), (257, 1, 2, 64), (290, 2, 1, 32)])
def test_lengths(T, n_seq, H, hd, dtype):
    say("relpos", dtype, "T=%d n_seq=%d H=%d hd=%d" % (T, n_seq, H, hd))
    Case(*line_index(T, 9), n_seq, H, hd, dtype, seed=120 + T).run()


@pytest.mark.parametrize("side,extra,n_seq,H,hd,dtype", [
    (7, False, 9, 3, 32, "bf16"), (7, True, 3, 2, 64, "f16"), (12, False, 2, 2, 32, "bf16"),
    (14, True, 1, 3, 64, "bf16"), (4, False, 33, 4, 32, "f16")])
def test_windows(side, extra, n_seq, H, hd, dtype):
    say("relpos window", side, extra, dtype)
    Case(*window_index(side, extra), n_seq, H, hd, dtype, seed=130).run()


@pytest.mark.parametrize("T,hd", [(49, 32), (49, 64), (20, 32), (100, 64), (197, 32), (230, 64), (261, 32)])
def test_labels_and_padding(T, hd):
    """Parts of a window, labels of every sign, sequences padded wholly and in part; padding
    tokens hold NaN and infinities."""
    say("relpos labels", T, hd)
    r = np.random.default_rng(T)
    region = r.integers(0, 3, (4, T))
    region[1, T // 2:] = -1
    region[2] = -7
    region[3, ::3] = np.iinfo(np.int32).min
    region[3, 1::3] = np.iinfo(np.int32).max

    def spoil(c):
        for n in range(c.n_seq):
            for i in np.flatnonzero(region[n % 4] < 0):
                bad = [np.nan, np.inf, -np.inf][i % 3]
                c.x[n * T + i] = bad
                c.g[n * T + i] = bad
                c.qkv[n * T + i] = bad
                c.dout[n * T + i] = bad
    c = Case(*line_index(T, 12), 6, 2, hd, "bf16", region=region, seed=140, edit=spoil)
    out, lse, dqkv, dtable = c.run()
    pad = torch.from_numpy(np.concatenate([region[n % 4] < 0 for n in range(6)])).cuda()
    assert not out[pad].any() and not dqkv[pad].any()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_masks_that_leave_nothing(dtype):
    """Index -1 (a causal order, a row and a column without pairs) and biases of -inf and of
    the type's lowest value."""
    T = 70
    idx, n = line_index(T, 20)
    idx[np.triu_indices(T, 1)] = -1
    idx[40] = -1
    idx[:, 3] = -1
    bad = {3: -np.inf, 4: LOWEST[dtype]}

    def edit(c):
        for b, v in bad.items():
            c.t[b] = v
            c.table[b] = v
    c = Case(idx, n, 3, 2, 32, dtype, seed=150, edit=edit)
    out, lse, dqkv, dtable = c.run()
    assert not out.view(3, T, -1)[:, 40].any() and bool((lse[:, :, 40] == -float("inf")).all())
    assert not dtable[list(bad)].any()


@pytest.mark.parametrize("dtype,value", [("bf16", -2.0 ** 30), ("bf16", -2.0 ** 100), ("bf16", 2.0 ** 60),
                                         ("f16", -60000.0), ("bf16", -2.0 ** 15), ("bf16", -16384.0)])
@pytest.mark.parametrize("T", [30, 49, 100, 240])
def test_rows_of_large_biases_alone(T, dtype, value):
    """Rows whose every pair has one large bias are as without it, beside rows where a few pairs
    have it: beyond 2^15 it counts as that."""
    idx, n = line_index(T, 9)
    idx[T // 2] = 8
    idx[3] = 8
    idx[:3] = np.minimum(idx[:3], 7)  # (rows without it)

    def edit(c):
        c.t[8] = np.clip(value, -2.0 ** 15, 2.0 ** 15)
        c.table[8] = value
    Case(idx, n, 3, 2, 32, dtype, seed=165, edit=edit).run()


def test_every_pair_masked():
    c = Case(np.full((40, 40), -1, np.int32), 5, 3, 2, 64, "bf16", seed=151)
    out, lse, dqkv, dtable = c.run()
    assert not out.any() and not dqkv.any() and not dtable.any()


@pytest.mark.parametrize("T,n_seq,H", [(100, 5, 3), (197, 90, 3), (70, 1, 1), (145, 257, 2), (240, 7, 2),
                                       (230, 40, 8)])
def test_many_sequences_and_heads(T, n_seq, H):
    """More and fewer sequences than workgroups: whole heads, parts of them, several heads to
    a workgroup; few and many tiles."""
    say("relpos sums", T, n_seq, H)
    idx, n = line_index(T, 7)
    c = Case(idx, n, 1, H, 32, "bf16", seed=156)
    # the same sequence n_seq times: dtable is n_seq times one's, dqkv repeats
    one_out, one_lse = c.forward()
    dq1, dt1 = c.grad(one_out, one_lse)
    rep = lambda t: t.repeat(n_seq, 1)
    qkv, dout = rep(c.qkv), rep(c.dout)
    lse = torch.empty((n_seq, H, T), device="cuda")
    out = lpv.relpos_attention(c.rp, c.table, qkv, n_seq, H, lse=lse, hd=32)
    dq, dt = lpv.relpos_attention_grad(c.rp, c.table, qkv, out, lse, dout, n_seq, H, hd=32)
    torch.cuda.synchronize()
    # (the kernels differ by the number of sequences, and with them the orders of sums: their
    # float32 differences, and the half steps that two roundings of nearly the same may differ by)
    for a, b in ((out, rep(one_out)), (dq, rep(dq1))):
        a, b = a.float(), b.float()
        assert float((a - b).abs().max()) <= 2 * U["bf16"] * float(b.abs().max())
    want = dt1.double() * n_seq
    err = (dt.double() - want).abs()
    # dt1 and dt are rounded once each, and dS is summed in float32, 2^-24 a term of at most
    # T^2 n_seq.  The gradients take D from the outputs as they were rounded: either's is off by
    # at most u (P |V| + |O|) <= 2.1 u P |V|, so the two D by twice the sum of |dO| times that,
    # in every sequence alike, which dS_ij takes P_ij times
    r = ft.relpos_attention(c.x, c.t, idx, 1, H, 32, dout=c.g)
    e_D = 2 * 2.1 * U["bf16"] * (np.abs(c.g) * r["abs_pv"]).reshape(T, H, 32).sum(2)
    e_t = np.zeros((n, H))
    for h in range(H):
        np.add.at(e_t[:, h], idx, r["P"][0, h] * e_D[:, h][:, None])
    bound = 2 * U["bf16"] * want.abs() + 2 ** -16 * T * n_seq + torch.from_numpy(n_seq * e_t).cuda()
    assert bool((err <= bound).all())


@pytest.mark.parametrize("T", [49, 100])
def test_large_biases_and_sharp_scores(T):
    def edit(c):
        c.t[2], c.t[5] = 60.0, -200.0
        c.table[2], c.table[5] = 60.0, -200.0
    Case(*line_index(T, 9), 2, 2, 64, "bf16", seed=152, q_std=3.0, edit=edit).run()


def test_strided_rows_and_neighbours_left_alone():
    """Row strides above the row, inputs and outputs inside larger tensors: what lies beside
    and behind the rows stays as it was."""
    c = Case(*window_index(6), 4, 3, 32, "bf16", seed=153)
    M, D = 4 * 36, 96
    ref = c.run()
    wide = torch.full((M + 3, 3 * D + 24), 5.0, dtype=torch.bfloat16, device="cuda")
    wide[:M, 8:8 + 3 * D] = c.qkv
    outs = torch.full((M + 3, D + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    grads = torch.full((M + 3, 3 * D + 16), 5.0, dtype=torch.bfloat16, device="cuda")
    gout = torch.full((M, D + 40), 5.0, dtype=torch.bfloat16, device="cuda")
    gout[:, 16:16 + D] = c.dout
    lse = torch.empty((4, 3, 36), device="cuda")
    dtable = torch.empty_like(c.table)
    out = lpv.relpos_attention(c.rp, c.table, wide[:M, 8:8 + 3 * D], 4, 3, out=outs[:M, :D], lse=lse,
                               hd=32)
    lpv.relpos_attention_grad(c.rp, c.table, wide[:M, 8:8 + 3 * D], out, lse, gout[:, 16:16 + D], 4, 3,
                              dqkv=grads[:M, 8:8 + 3 * D], dtable=dtable, hd=32)
    torch.cuda.synchronize()
    for a, b in ((out, ref[0]), (lse, ref[1]), (grads[:M, 8:8 + 3 * D], ref[2]), (dtable, ref[3])):
        assert torch.equal(a, b)
    assert (outs[:M, D:] == 5).all() and (outs[M:] == 5).all() and (grads[M:] == 5).all()
    assert (grads[:M, :8] == 5).all() and (grads[:M, 8 + 3 * D:] == 5).all()


@pytest.mark.parametrize("T", [49, 80])
def test_same_bits_each_time_and_on_another_stream(T):
    c = Case(*line_index(T), 40, 3, 32, "f16", seed=154)
    first = [t.clone() for t in c.run()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out, lse = c.forward()
        again = (out, lse) + c.grad(out, lse)
    s.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    ws = torch.empty(lpv.relpos_workspace_size(c.rp, 40, 3, True), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    dqkv, dtable = c.grad(first[0], first[1], workspace=ws.fill_(255), stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(dqkv, first[2]) and torch.equal(dtable, first[3])
    if lpv.relpos_workspace_size(c.rp, 40, 3):
        with pytest.raises(ValueError):  # torch's allocator would hand the workspace out too early
            c.forward(stream=s)


@pytest.mark.parametrize("T", [49, 130])
def test_graph_replays(T):
    """Forward and gradient captured together: replays, each after eager work on other
    values, give the eager result."""
    c = Case(*line_index(T), 6, 2, 64, "bf16", seed=155)
    ref = [t.clone() for t in c.run()]
    keep = c.qkv.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = c.forward()
        res = (out, lse) + c.grad(out, lse)
    for _ in range(3):
        c.qkv.mul_(-0.5)
        o, l = c.forward()
        c.grad(o, l)
        c.qkv.copy_(keep)
        for t in res:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(res, ref):
            assert torch.equal(a, b)


def test_empty_batch():
    c = Case(*window_index(3), 0, 2, 32, "bf16")
    out, lse = c.forward()
    dqkv, dtable = c.grad(out, lse, dtable=torch.full((25, 2), 3.0, dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    assert out.shape == (0, 64) and dqkv.shape == (0, 192) and not dtable.any()


def test_more_sequences_than_one_grid_dimension_holds():
    # one token each: the weight is 1, the output V, dV = dO, dQ = dK = 0
    n = 2 ** 22 + 7
    say("relpos sequences", n)
    rp = lpv.relpos(torch.zeros((1, 1), dtype=torch.int32, device="cuda"), 1)
    table = torch.ones((1, 1), dtype=torch.bfloat16, device="cuda")
    qkv = torch.randn((n, 96), dtype=torch.bfloat16, device="cuda")
    dout = torch.randn((n, 32), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((n, 1, 1), device="cuda")
    out = lpv.relpos_attention(rp, table, qkv, n, 1, lse=lse, hd=32)
    assert torch.equal(out, qkv[:, 64:])
    dqkv, dtable = lpv.relpos_attention_grad(rp, table, qkv, out, lse, dout, n, 1, hd=32)
    assert torch.equal(dqkv[:, 64:], dout)
    # dP and D are the same 32 products, summed in float32 in two orders; P is 1 to 2^-20
    most = 64 * 2.0 ** -24 * float((dout.float() * qkv[:, 64:].float()).abs().sum(1).max())
    assert float(dqkv[:, :64].abs().max()) <= most * float(qkv.abs().max()) / 32 ** 0.5
    assert float(dtable.abs().max()) <= most * n


@pytest.mark.parametrize("bad", [5, -2, 2 ** 31 - 1, -2 ** 31])
def test_index_outside_the_table_is_refused(bad):
    idx = torch.zeros((6, 6), dtype=torch.int32, device="cuda")
    idx[2, 4] = bad
    with pytest.raises(lpv.LpvError, match=r"index\[2\]\[4\]"):
        lpv.relpos(idx, 5)


def test_refusals_of_the_binding():
    c = Case(*window_index(3), 2, 2, 32, "bf16")
    out, lse = c.forward()
    for kw in ({"region": torch.zeros((1, 8), dtype=torch.int32, device="cuda")},
               {"region": torch.zeros((1, 9), dtype=torch.int64, device="cuda")},
               {"out": out[:, :32]}, {"lse": lse.double()}, {"out": out.float()},
               {"region": torch.zeros((1, 9), dtype=torch.int32)}):
        with pytest.raises((ValueError, TypeError)):
            lpv.relpos_attention(c.rp, c.table, c.qkv, 2, 2, hd=32, **kw)
    with pytest.raises(ValueError):
        lpv.relpos_attention(c.rp, c.table[:8], c.qkv, 2, 2, hd=32)
    with pytest.raises(lpv.LpvError):
        c.forward(out=c.qkv[:, :64])  # overlaps its input
    with pytest.raises(lpv.LpvError):
        c.grad(out, lse, dqkv=c.qkv)
    with pytest.raises(lpv.LpvError):
        c.grad(out, lse, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_each_kernel_is_reached():
    """The rules' sides: windows up to 64 tokens, scores in one pass up to 224, one or two waves
    to a tile behind that, the sequences' sums folded by 1 or 16 threads."""
    def names(T, n_seq, H):
        c = Case(*line_index(T, 9), 1, H, 32, "bf16", seed=157)
        qkv, dout = c.qkv.repeat(n_seq, 1), c.dout.repeat(n_seq, 1)
        lse = torch.empty((n_seq, H, T), device="cuda")
        res = []

        def calls():
            res.append(lpv.relpos_attention(c.rp, c.table, qkv, n_seq, H, lse=lse, hd=32))
            lpv.relpos_attention_grad(c.rp, c.table, qkv, res[-1], lse, dout, n_seq, H, hd=32)
        return {n.replace("lpv::(anonymous namespace)::", "").replace(" ", "") for n in kernels(calls, args=True)}
    one, two = "Shape<4,1>", "Shape<2,2>"
    for T, n_seq, H, there, absent in (
            (32, 40, 2, ("window_fwd<2,32,1", "window_grad<2,32,1", "fold<16>"), ("bias",)),
            (64, 3, 2, ("window_fwd<2,32,2", "window_grad<2,32,2", "fold<1>"), ("bias", "mid_grad")),
            (65, 3, 2, ("k_relpos_fwd<2,32", two, "mid_grad", "bias<2,0>"), ("window", "bias<2,32>")),
            (140, 80, 4, ("k_relpos_fwd<2,32", "Shape<3,1>", "mid_grad"), ("window", one, two)),
            (224, 70, 4, ("k_relpos_fwd<2,32", one, "mid_grad"), ("window", "k_relpos_grad")),
            (225, 2, 2, ("k_relpos_grad<2,32", two, "bias<2,0>", "bias<2,32>", "pairs"), (one, "mid_grad")),
            (225, 16, 4, ("k_relpos_grad<2,32", one, two, "bias<2,0>", "bias<2,32>"), ("mid_grad",))):
        got = names(T, n_seq, H)
        for n in there:
            assert any(n in g for g in got), (T, n, got)
        for n in absent:
            assert not any(n in g for g in got), (T, n, got)
    c = Case(*window_index(16), 1, 1, 32, "bf16", seed=157)  # (more buckets than tokens)
    assert not any("pairs" in n for n in kernels(lambda: c.grad(*c.forward())))


@pytest.mark.parametrize("T,n_seq,H,labels", [(230, 20, 4, True), (230, 20, 4, False), (225, 37, 2, True)])
def test_labels_with_many_tiles(T, n_seq, H, labels):
    """One wave to a tile in the general gradients, with and without labels."""
    region = None
    if labels:
        region = np.random.default_rng(T).integers(0, 2, (5, T))
        region[1, T // 2:] = -1
        region[4] = -1
        region[3] = 8
    Case(*line_index(T, 12), n_seq, H, 32, "bf16", region=region, seed=158).run()


@pytest.mark.parametrize("T,n_seq,H,hd,labels", [(140, 80, 4, 32, True), (170, 70, 4, 64, False),
                                                 (81, 130, 4, 64, True), (200, 60, 4, 32, True)])
def test_forward_with_many_tiles(T, n_seq, H, hd, labels):
    """Three and four tiles to a workgroup, one wave each."""
    region = None
    if labels:
        region = np.random.default_rng(T).integers(0, 2, (3, T))
        region[1, T // 2:] = -1
        region[2] = 8
    Case(*line_index(T, 12), n_seq, H, hd, "bf16", region=region, seed=164).run()


@pytest.mark.parametrize("T,n_buckets", [(60, 20000), (130, 20000), (130, 12288), (130, 12289), (240, 65535)])
def test_many_buckets(T, n_buckets):
    """Tables around and past the size whose column LDS holds; most buckets without a pair."""
    idx = np.random.default_rng(T).integers(-1, n_buckets, (T, T)).astype(np.int32)
    idx[5, 5] = n_buckets - 1
    c = Case(idx, n_buckets, 2, 2, 32, "bf16", seed=159)
    dtable = c.run()[3]
    unused = np.ones(n_buckets, bool)
    unused[idx[idx >= 0]] = False
    assert not dtable[torch.from_numpy(unused).cuda()].any()


def test_longest_sequence():
    say("relpos T=2048")
    Case(*line_index(2048, 64), 1, 1, 32, "bf16", seed=160).run()


@pytest.mark.parametrize("T,n_seq", [(49, 12), (100, 6), (260, 3)])
def test_rows_past_32_bits(T, n_seq):
    """Rows at the largest stride, so that the last lie over 2^31 elements behind the first:
    the same bits as packed."""
    say("relpos strides", T, n_seq)
    c = Case(*line_index(T, 9), n_seq, 2, 32, "bf16", seed=161)
    ref = c.forward()
    ref += c.grad(*ref)
    M, ld = n_seq * T, 2 ** 22

    def wide(t):
        w = torch.empty(M * ld, dtype=torch.bfloat16, device="cuda").as_strided((M, t.shape[1]), (ld, 1))
        return w.copy_(t)
    assert (M - 1) * ld > 2 ** 31
    out = wide(torch.zeros_like(ref[0]))
    lse = torch.empty_like(ref[1])
    qkv, dqkv = wide(c.qkv), wide(torch.zeros_like(c.qkv))
    lpv.relpos_attention(c.rp, c.table, qkv, n_seq, 2, out=out, lse=lse, hd=32)
    dout = wide(c.dout)
    dtable = lpv.relpos_attention_grad(c.rp, c.table, qkv, out, lse, dout, n_seq, 2, dqkv=dqkv, hd=32)[1]
    torch.cuda.synchronize()
    for a, b in ((out, ref[0]), (lse, ref[1]), (dqkv, ref[2]), (dtable, ref[3])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [49, 130, 230])
def test_two_streams_share_a_handle(T):
    """Calls at once on two streams, each with its own workspace."""
    a = Case(*line_index(T, 9), 30, 3, 32, "bf16", seed=162)
    b = Case(*line_index(T, 9), 30, 3, 32, "bf16", seed=163)
    b.rp = a.rp
    ref = [c.forward() for c in (a, b)]
    ref = [r + c.grad(*r) for c, r in zip((a, b), ref)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(4):
        for i, c in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                r = c.forward()
                got[i].append(r + c.grad(*r))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            for x, y in zip(r, ref[i]):
                assert torch.equal(x, y)


@pytest.mark.parametrize("T,n_seq,H", [(40, 3, 2), (230, 3, 2), (300, 2, 2), (520, 1, 1), (290, 17, 4)])
def test_few_buckets_keep_the_tables_gradient(T, n_seq, H):
    """Every bucket takes many pairs of each row, so an error of D would add up along the row: the
    sums take D without the rounding of the outputs.  What is left: float32, and the rounding."""
    say("relpos few buckets", T, n_seq, H)
    c = Case(*line_index(T, 4), n_seq, H, 32, "bf16", seed=166)
    out, lse = c.forward()
    dtable = c.grad(out, lse)[1]
    torch.cuda.synchronize()
    r = ft.relpos_attention(c.x, c.t, c.idx, n_seq, H, 32, dout=c.g)
    # a weight is off by f (the module's text); D, as the weights have it, by f and the sums'
    # (T + 32) 2^-24 of sum_j P |dP|; twice that for D's two places
    f = 2 * 34 * 2.0 ** -24 * r["abs_s"] + 2.0 ** -20 + 2.0 ** -22 * (1 + np.abs(r["lse"]))
    P, dP, B = r["P"], r["dP"], r["abs_dP"]
    size = (P * B).sum(3)
    e = P * ((f + (T + 40) * 2.0 ** -24)[..., None] * (B + 3 * size[..., None]))
    e_t = np.zeros(c.t.shape)
    pairs = (e + (n_seq * T + 8) * 2.0 ** -24 * P * (B + size[..., None])).sum(0)
    for h in range(H):
        np.add.at(e_t[:, h], c.idx, pairs[h])
    c.within(f64(dtable), r["dtable"], 1.02 * e_t + U["bf16"] * np.abs(r["dtable"]), "dtable")


def class_index(s):
    """window_index(s, True): the first row gives one bucket all its pairs but one."""
    return window_index(s, True)


def diagonal_index(T):
    return 1 - np.eye(T, dtype=np.int32), 2


def between_steps(c):
    """Values of 1 and, a quarter of them, one step of the type above: outputs lie a quarter of a
    step above 1 and are rounded to it in every row, so that with gradients around 1 all rows' dout .
    out are too small by about as much (bf16: 2^-9 of their size, far over what float32 leaves)."""
    step, D = 2 * U[c.dtype], c.H * c.hd
    r = np.random.default_rng(175)
    c.x[:, 2 * D:] = 1 + step * (r.random((len(c.x), D)) < 0.25)
    c.g[:] = 1 + 0.25 * r.integers(-2, 3, c.g.shape)
    c.qkv[:, 2 * D:] = torch.from_numpy(c.x[:, 2 * D:])
    c.dout[:] = torch.from_numpy(c.g)


def table_bound(c, n_seq, H, r):
    """What float32 leaves of the table's gradient (as in the test of few buckets): a weight is
    off by f; D, as the weights have it, by f and the sums' (T + 32) 2^-24 of sum_j P |dP|; twice
    that for D's two places."""
    T, hd = c.T, c.hd
    f = 2 * (hd + 2) * 2.0 ** -24 * r["abs_s"] + 2.0 ** -20 + 2.0 ** -22 * (1 + np.abs(r["lse"]))
    P, B = r["P"], r["abs_dP"]
    size = (P * B).sum(3)
    e = P * ((f + (T + hd + 8) * 2.0 ** -24)[..., None] * (B + 3 * size[..., None]))
    pairs = (e + (n_seq * T + 8) * 2.0 ** -24 * P * (B + size[..., None])).sum(0)
    e_t = np.zeros(c.t.shape)
    for h in range(H):
        np.add.at(e_t[:, h], c.idx, pairs[h])
    return 1.02 * e_t + U[c.dtype] * np.abs(r["dtable"]) + TINY[c.dtype]


@pytest.mark.parametrize("index,T,n_seq,H,hd,dtype", [
    ("line", 65, 5, 2, 32, "bf16"), ("line", 100, 3, 2, 32, "bf16"), ("line", 100, 70, 4, 64, "f16"),
    ("line", 160, 2, 3, 64, "bf16"), ("line", 197, 9, 2, 32, "f16"), ("line", 224, 2, 2, 64, "bf16"),
    ("diagonal", 70, 3, 2, 64, "bf16"), ("diagonal", 200, 4, 2, 32, "bf16"), ("diagonal", 260, 3, 2, 32, "f16"),
    ("distances", 130, 4, 2, 32, "bf16"), ("distances", 300, 4, 2, 32, "bf16")])
def test_crowded_rows_keep_the_tables_gradient(index, T, n_seq, H, hd, dtype):
    """Every row gives a bucket many of its pairs, or a few: an error of D would add up."""
    say("relpos crowded rows", index, T, n_seq, H, hd, dtype)
    idx, n = {"line": lambda: line_index(T, 4), "diagonal": lambda: diagonal_index(T),
              "distances": lambda: (np.abs(line_index(T, 2 * T)[0] - T).astype(np.int32), T + 1)}[index]()
    c = Case(idx, n, n_seq, H, hd, dtype, seed=170, q_std=0.3, edit=between_steps)
    out, lse = c.forward()
    dqkv, dtable = c.grad(out, lse)
    torch.cuda.synchronize()
    c.check(out, lse, dqkv, dtable)
    r = ft.relpos_attention(c.x, c.t, c.idx, n_seq, H, hd, dout=c.g)
    c.within(f64(dtable), r["dtable"], table_bound(c, n_seq, H, r), "dtable")


@pytest.mark.parametrize("side,n_seq,H,hd,dtype", [
    (8, 6, 2, 32, "bf16"), (10, 40, 3, 64, "bf16"), (14, 8, 3, 64, "bf16"), (14, 3, 2, 32, "f16"),
    (15, 2, 2, 32, "bf16"), (17, 8, 2, 32, "bf16"), (23, 2, 1, 64, "f16")])
def test_the_class_tokens_buckets_keep_their_gradient(side, n_seq, H, hd, dtype):
    """The class token's row is one bucket, in a table of many more: its gradient is what little is
    left of a row that sums to zero.  (Its label apart, the same with padding.)"""
    idx, n = class_index(side)
    T = len(idx)
    say("relpos class token", side, n_seq, H, hd, dtype)
    pad = np.zeros((2, T), np.int64)
    pad[1, T - T // 3:] = -1
    for region in (None, pad):
        c = Case(idx, n, n_seq, H, hd, dtype, region=region, seed=171, q_std=0.3, edit=between_steps)
        out, lse = c.forward()
        dtable = c.grad(out, lse)[1]
        torch.cuda.synchronize()
        r = ft.relpos_attention(c.x, c.t, c.idx, n_seq, H, hd, region=region, dout=c.g)
        r["lse"] = np.where(r["lse"] == -np.inf, 0.0, r["lse"])
        bound = table_bound(c, n_seq, H, r)
        row = [n - 3, n - 1]  # the buckets of the first row
        c.within(f64(dtable)[row], r["dtable"][row], bound[row], "dtable's class token")


def test_the_pairs_launch_is_for_crowded_rows():
    """Past 224 tokens: a class token's row is one bucket, though the table is larger than the row."""
    c = Case(*class_index(16), 1, 1, 32, "bf16", seed=172)
    assert any("pairs" in n for n in kernels(lambda: c.grad(*c.forward())))


def test_one_row_of_any_stride():
    """A matrix of one row has no stride to speak of: that of a slice of a wider tensor is not
    looked at."""
    c = Case(np.zeros((1, 1), np.int32), 1, 1, 2, 32, "bf16", seed=173)
    ref = c.run()
    D = 64
    room = torch.full((2, 3 * D + 9), 5.0, dtype=torch.bfloat16, device="cuda")
    far = torch.full((1, 2 ** 22 + 24), 5.0, dtype=torch.bfloat16, device="cuda")
    qkv, dqkv = room[:1, :3 * D], far[:, 8:8 + 3 * D]
    qkv.copy_(c.qkv)
    lse = torch.empty((1, 2, 1), device="cuda")
    out = lpv.relpos_attention(c.rp, c.table, qkv, 1, 2, lse=lse, hd=32)
    dtable = lpv.relpos_attention_grad(c.rp, c.table, qkv, out, lse, c.dout, 1, 2, dqkv=dqkv, hd=32)[1]
    torch.cuda.synchronize()
    for a, b in zip((out, lse, dqkv, dtable), ref):
        assert torch.equal(a, b)
    assert (far[:, :8] == 5).all() and (far[:, 8 + 3 * D:] == 5).all()
