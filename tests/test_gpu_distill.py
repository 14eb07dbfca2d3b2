"""GPU parity of the distillation loss and its gradient against the float64 oracle.

The tolerances are bounds on each element.  u is half a step of the element type (2^-24
fp32, 2^-11 fp16, 2^-8 bf16).  With d = (z_max - z) / tau, a weight exp(-d) is off by
e(d) = 2^-22 (2 + 2 d) relative (the difference, the product with log2(e) / tau, its own
rounding, exp2), a sum of them by the same and by its additions, at most 2^-16 (128 terms
a thread and the tree over them; 2^-18 for the teacher's up to 1024 entries).  A log is off
by that relative error and by 2^-22 of what its terms z / tau and max / tau hold (rows cut
into chunks add those, instead of their difference)."""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from gpu_util import dev, f64, kernels, say
from oracle import finetune as ft
from paper_2407_02068_amd import lpv

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -126}  # (a result below 2^-126 may flush)
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


class Case:
    def __init__(self, M, V, k, dtype, tau=1.0, seed=160, std=3.0, ragged=False, edit=None):
        self.M, self.V, self.k, self.dtype, self.tau = M, V, k, dtype, tau
        r = np.random.default_rng(seed)
        a = wl.quantize(r.normal(0, std, (M, V)).astype(np.float32), dtype)
        self.z = oracle.decode(a, dtype).reshape(M, V)
        self.ids = np.stack([r.permutation(V)[:k] if k <= V else r.integers(0, V, k) for _ in range(M)]
                            ).astype(np.int32).reshape(M, k)
        self.t = (8 - np.cumsum(r.exponential(0.4, (M, k)), 1)).astype(np.float32)
        if ragged:
            self.ids[np.arange(k)[None, :] >= r.integers(0, k + 1, (M, 1))] = -1
        self.g = r.normal(0, 1, M).astype(np.float32)
        if edit:
            edit(self)
        pad = (V + 15) // 16 * 16
        wide = torch.full((M, pad), 3.0, dtype=TORCH[dtype], device="cuda")
        wide[:, :V] = torch.from_numpy(self.z).cuda().to(TORCH[dtype])
        self.logits = wide[:, :V]
        self.dev = (torch.from_numpy(self.ids).cuda(), torch.from_numpy(self.t).cuda())
        self.dloss = torch.from_numpy(self.g).cuda()

    def check(self, loss, dlogits=None):
        tau, u = self.tau, U[self.dtype]
        with np.errstate(invalid="ignore"):
            want, dwant = ft.distill(self.z, self.ids, self.t, tau, self.g.astype(np.float64))
        got = f64(loss)
        e_loss, e_d = np.zeros(self.M), np.zeros((self.M, self.V))
        for r in range(self.M):
            use = np.flatnonzero((self.ids[r] >= 0) & (self.ids[r] < self.V) & (self.t[r] > -np.inf))
            if not len(use):
                continue
            z, t, at = self.z[r] / tau, self.t[r, use].astype(np.float64) / tau, self.ids[r, use]
            fin = np.isfinite(z)
            top = z[fin].max()
            d = np.where(fin, top - z, 0.0)
            p = np.where(fin, np.exp(-d), 0.0)
            p /= p.sum()
            q = np.exp(t - t.max())
            q /= q.sum()
            dq = t.max() - t
            e_sum = (p * 2.0 ** -22 * (2 + 2 * d)).sum() + 2.0 ** -16
            e_qs = (q * 2.0 ** -22 * (2 + 2 * dq)).sum() + 2.0 ** -18
            size = np.abs(z[fin]).max()
            e_q = 2.0 ** -22 * (2 + 2 * dq) + e_qs
            Q, EQ = np.zeros(self.V), np.zeros(self.V)
            np.add.at(Q, at, q)
            np.add.at(EQ, at, q * (e_q + (len(use) + 1) * 2.0 ** -24))
            w = abs(self.g[r]) * tau
            e_d[r] = w * (p * (2.0 ** -22 * (3 + 2 * d) + e_sum) + EQ + 2.0 ** -23 * np.abs(p - Q))
            log_q, log_p = -dq - np.log(np.exp(-dq).sum()), -d[at] - np.log(np.exp(-d[fin]).sum())
            have = (q > 0) & fin[at]
            term = np.abs(log_q - log_p)
            e_log = e_qs + e_sum + 2.0 ** -22 * (dq + d[at] + np.abs(log_q) + np.abs(log_p) + 4 * size + 2)
            e_loss[r] = tau ** 2 * (q * (e_q * term + e_log + 2.0 ** -18 * (term + size)))[have].sum()
        inf = ~np.isfinite(want)
        assert np.array_equal(got[inf], want[inf])
        self.within(got[~inf], want[~inf], e_loss[~inf] + 2.0 ** -22 * np.abs(want[~inf]), "loss")
        if dlogits is not None:
            self.within(f64(dlogits), dwant, e_d + u * np.abs(dwant) + TINY[self.dtype], "dlogits")

    @staticmethod
    def within(got, want, bound, what):
        assert np.isfinite(got).all(), what + " is not finite"
        worst = float((np.abs(got - want) / (bound + 1e-37)).max()) if got.size else 0.0
        say("  %s: at most %.2f of its bound (mean bound %.1e, mean value %.1e)"
            % (what, worst, bound.mean() if got.size else 0, np.abs(want).mean() if got.size else 0))
        assert worst <= 1.0, "%s: %.3g times its bound" % (what, worst)

    def run(self, **kw):
        alone = lpv.distill_loss(self.logits, *self.dev, self.tau)
        loss, d = lpv.distill_grad(self.logits, *self.dev, self.tau, self.dloss, **kw)
        torch.cuda.synchronize()
        self.check(loss, d)
        assert torch.equal(alone, loss) or bool(torch.isnan(loss).any())
        return loss, d


SHAPES = [
    # (rows, classes, entries): one class; around a chunk's edge; a wave's rows
    (3, 1, 1), (5, 2, 3), (9, 7, 4), (9, 8, 8), (9, 9, 9), (130, 1000, 16), (33, 1009, 64),
    (2, 2047, 64), (3, 2049, 5), (2, 4095, 17),
    # a workgroup's: more entries than a wave's lanes, longer rows
    (5, 70, 65), (4, 1000, 1024), (3, 5000, 100), (140, 9000, 33), (130, 21841, 64),
    # 512 and 1024 threads, and rows cut into chunks
    (130, 40003, 20), (130, 65535, 70), (2, 100000, 200), (1, 131072, 128), (1, 131101, 1), (1, 30001, 9)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,V,k", SHAPES)
def test_shapes(M, V, k, dtype):
    say("distill", dtype, "M=%d V=%d k=%d" % (M, V, k))
    Case(M, V, k, dtype, tau=2.0, seed=160 + V % 97, ragged=M > 4).run()


def test_each_kernel_is_reached():
    """The rule's sides: a wave, a workgroup of 256, 512 and 1024, and chunks."""
    def names(M, V, k, dtype):
        c = Case(M, V, k, dtype)
        return kernels(lambda: lpv.distill_grad(c.logits, *c.dev, 1.0, c.dloss), args=True)
    for M, V, k, dtype, want in ((4, 4096, 64, "bf16", "k_distill_row<2, 64, 8>"),
                                 (4, 2048, 64, "f32", "k_distill_row<0, 64, 8>"),
                                 (4, 1000, 65, "bf16", "k_distill_row<2, 256, 1>"),
                                 (128, 32768, 4, "f16", "k_distill_row<1, 256, 16>"),
                                 (128, 40000, 4, "f16", "k_distill_row<1, 512, 12>"),
                                 (128, 100000, 4, "bf16", "k_distill_row<2, 1024, 16>"),
                                 (128, 65540, 4, "f32", "k_distill_join<0>"),
                                 (127, 65545, 4, "bf16", "k_distill_join<2>"),
                                 (127, 65536, 4, "bf16", "k_distill_row<2, 512, 16>")):
        assert want in names(M, V, k, dtype)


@pytest.mark.parametrize("V,M", [(1000, 6), (9000, 6), (120000, 2)])
def test_the_same_class_twice(V, M):
    def edit(c):
        c.ids[0] = 5                       # one class takes everything
        c.ids[1] = c.ids[1] % 7            # a few classes
        c.ids[-1, ::2] = c.ids[-1, 1::2]   # pairs
    for k in (4, 64, 200):
        Case(M, V, k, "f32", tau=1.5, seed=170, edit=edit).run()


@pytest.mark.parametrize("V,M", [(1000, 8), (9000, 8), (120000, 8)])
def test_entries_that_are_none(V, M):
    def edit(c):
        c.ids[0] = -1
        c.ids[1] = V
        c.ids[2, ::2] = np.iinfo(np.int32).min
        c.ids[3, 1:] = np.iinfo(np.int32).max
        c.t[4] = -np.inf
        c.t[5, 3:] = -np.inf
        c.z[0] = np.nan  # no entries: whatever the row holds, loss and gradient are zero
    c = Case(M, V, 12, "bf16", seed=171, edit=edit)
    loss, d = lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss)
    torch.cuda.synchronize()
    for r in (0, 1, 4):
        assert loss[r] == 0 and not d[r].any()
    c.z[0] = 0
    c.check(loss, d)


@pytest.mark.parametrize("V,M", [(1000, 5), (9000, 5), (120000, 3)])
def test_classes_left_out(V, M):
    """Logits of -inf: no probability; under one of the teacher's classes an infinite loss
    with a finite gradient."""
    def edit(c):
        keep = c.ids[0].copy()
        c.z[0, ::3] = -np.inf
        c.z[0, keep] = 1.0
        c.z[1] = -np.inf
        c.z[1, c.ids[1]] = 0.5
        c.z[2, c.ids[2, 3]] = -np.inf
    c = Case(M, V, 10, "f32", tau=3.0, seed=172, edit=edit)
    loss, d = c.run()
    assert bool(torch.isinf(loss[2])) and bool(torch.isfinite(d).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tau,std", [(1e-3, 0.01), (0.25, 10.0), (1000.0, 50.0), (1.0, 1000.0)])
def test_temperatures_and_large_logits(dtype, tau, std):
    Case(6, 777, 20, dtype, tau=tau, seed=173, std=std).run()
    Case(1, 33000, 20, dtype, tau=tau, seed=174, std=std).run()


@pytest.mark.parametrize("M,V,k", [(9, 1000, 16), (5, 21841, 30), (2, 120000, 100)])
def test_in_place_strides_and_neighbours(M, V, k):
    """dlogits in the logits' own place; row strides above the row; the padding columns are
    zero, what lies behind them and beside the entries stays."""
    c = Case(M, V, k, "bf16", seed=175)
    loss, d = c.run()
    wide = d.as_strided((M, (V + 15) // 16 * 16), (d.stride(0), 1))
    assert not wide[:, V:].any()
    room = torch.full((M + 1, V // 8 * 8 + 64), 9.0, dtype=torch.bfloat16, device="cuda")
    room[:M, 8:8 + V] = c.logits
    z = room[:M, 8:8 + V]
    ids = torch.full((M, k + 5), 1, dtype=torch.int32, device="cuda")
    t = torch.full((M, k + 5), 50.0, device="cuda")
    ids[:, 2:2 + k], t[:, 2:2 + k] = c.dev
    keep = torch.full((M + 2,), 4.0, device="cuda")
    got, same = lpv.distill_grad(z, ids[:, 2:2 + k], t[:, 2:2 + k], c.tau, c.dloss, loss=keep[1:-1],
                                 dlogits=z)
    torch.cuda.synchronize()
    assert same is z and torch.equal(z, d) and torch.equal(got, loss)
    assert keep[0] == 4 and keep[-1] == 4
    assert (room[:, :8] == 9).all() and (room[:, 8 + V:] == 9).all() and (room[M] == 9).all()


def test_dloss_left_out_is_one():
    c = Case(4, 300, 7, "f32", seed=176)
    c.g[:] = 1
    loss, d = lpv.distill_grad(c.logits, *c.dev, c.tau)
    c.check(loss, d)


@pytest.mark.parametrize("M,V", [(40, 1000), (3, 50000)])
def test_stream_and_graph(M, V):
    c = Case(M, V, 20, "f16", seed=177)
    ref = [t.clone() for t in c.run()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        res = lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss)
    keep = c.logits.clone()
    for _ in range(3):
        c.logits.mul_(0.5)
        lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss)
        c.logits.copy_(keep)
        for t in res:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b, o in zip(res, ref, other):
            assert torch.equal(a, b) and torch.equal(o, b)


def test_no_rows_and_many_rows():
    z = torch.empty((0, 32), device="cuda")
    loss, d = lpv.distill_grad(z, torch.empty((0, 3), dtype=torch.int32, device="cuda"),
                               torch.empty((0, 3), device="cuda"), 1.0)
    assert loss.shape == (0,) and d.shape == (0, 32)
    # more workgroups than a row of the grid holds; two classes, the teacher sure of one:
    # with equal logits the loss is ln 2, the gradient (-1/2, 1/2)
    M = 2 ** 22 + 9
    say("distill rows", M)
    z = torch.zeros((M, 8), dtype=torch.bfloat16, device="cuda")[:, :2]
    ids = torch.zeros((M, 1), dtype=torch.int32, device="cuda")
    loss, d = lpv.distill_grad(z, ids, torch.ones((M, 1), device="cuda"), 1.0)
    assert float((loss - np.log(2)).abs().max()) <= 2.0 ** -21
    assert (d[:, 0] == -0.5).all() and (d[:, 1] == 0.5).all()


def test_refusals_of_the_binding():
    c = Case(4, 100, 5, "f32", seed=178)
    ids, t = c.dev
    for args in ((c.logits.double(), ids, t), (c.logits, ids.long(), t), (c.logits, ids, t.half()),
                 (c.logits, ids[:3], t), (c.logits, ids, t[:, :3]), (c.logits.cpu(), ids, t),
                 (c.logits, ids.cpu(), t), (c.logits, ids, t[:, ::2])):
        with pytest.raises((ValueError, TypeError)):
            lpv.distill_loss(*args, 1.0)
    for kw in ({"dloss": c.dloss[:2]}, {"dloss": c.dloss.double()}, {"loss": c.dloss.half()},
               {"dlogits": c.logits[:, :50]}, {"dlogits": c.logits.half()}):
        with pytest.raises((ValueError, TypeError)):
            lpv.distill_grad(c.logits, ids, t, 1.0, **kw)
    with pytest.raises(lpv.LpvError):
        lpv.distill_loss(c.logits, ids, t, 0.0)
    with pytest.raises(lpv.LpvError):
        lpv.distill_loss(c.logits, ids, t, float("nan"))


@pytest.mark.parametrize("M,V,k,dtype", [(2, 2 ** 22, 64, "bf16"), (1, 2 ** 22 - 5, 1000, "f16")])
def test_the_widest_rows(M, V, k, dtype):
    say("distill", dtype, "M=%d V=%d k=%d" % (M, V, k))
    Case(M, V, k, dtype, seed=180).run()


def test_rows_past_32_bits():
    """Rows at the largest stride: the last lie over 2^31 elements behind the first."""
    M, V, ld = 600, 1003, 2 ** 22
    c = Case(M, V, 9, "bf16", seed=181, ragged=True)
    loss, d = lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss)

    def wide():
        return torch.empty(M * ld, dtype=torch.bfloat16, device="cuda").as_strided((M, 1008), (ld, 1))
    assert (M - 1) * ld > 2 ** 31
    z, dz = wide(), wide()
    z[:, :V] = c.logits
    got, same = lpv.distill_grad(z[:, :V], *c.dev, c.tau, c.dloss, dlogits=dz)
    torch.cuda.synchronize()
    assert same is dz and torch.equal(got, loss) and torch.equal(dz[:, :V], d) and not dz[:, V:].any()


@pytest.mark.parametrize("M", [1, 3])
def test_gradient_with_padding_columns(M):
    """dlogits wider than the classes: its padding is cleared; in place too."""
    c = Case(M, 1003, 9, "bf16", seed=182)
    loss, d = lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss)
    wide = torch.full((M, 1024), 5.0, dtype=torch.bfloat16, device="cuda")
    lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss, dlogits=wide[:, :1016])
    torch.cuda.synchronize()
    assert torch.equal(wide[:, :1003], d) and not wide[:, 1003:1016].any() and (wide[:, 1016:] == 5).all()
    wide[:, :1003] = c.logits
    lpv.distill_grad(wide[:, :1003], *c.dev, c.tau, c.dloss, dlogits=wide)
    torch.cuda.synchronize()
    assert torch.equal(wide[:, :1003], d) and not wide[:, 1003:].any()
    for bad in (wide[:, :1000], wide[0], 3):
        with pytest.raises(ValueError):
            lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss, dlogits=bad)


def test_two_streams():
    cases = [Case(6, 131101, 30, "bf16", seed=183), Case(6, 131101, 30, "bf16", seed=184)]
    ref = [lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(4):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                got[i].append(lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert torch.equal(r[0], ref[i][0]) and torch.equal(r[1], ref[i][1])


@pytest.mark.parametrize("M,V,k,dtype,tau,offset", [
    # rows in a wave's, a workgroup's and 1024 threads' registers, and rows cut into chunks
    (6, 777, 20, "f32", 1.0, 30000.0), (6, 9000, 64, "f32", 2.0, -30000.0), (130, 60000, 30, "f32", 1.0, 30000.0),
    (3, 70000, 64, "f32", 1.0, 30000.0), (2, 70001, 9, "f32", 4.0, -30000.0), (1, 131072, 128, "f32", 0.5, 1000.0),
    (3, 70000, 64, "f16", 1.0, 1500.0), (6, 777, 20, "f16", 1.0, 1500.0)])
def test_a_common_offset_of_the_logits_costs_nothing(M, V, k, dtype, tau, offset):
    """p does not change with it, and the kernels take differences of the row's logits only: the
    loss's error is made of their sizes, |log q| and d = (z_max - z) / tau, not of z's."""
    def edit(c):
        a = wl.quantize((c.z + offset).astype(np.float32), dtype)
        c.z = oracle.decode(a, dtype).reshape(M, V)
    c = Case(M, V, k, dtype, tau=tau, seed=186, std=1.0, edit=edit)
    # (the teacher's logits are the student's own, but for a little: a loss near 0)
    c.t = np.take_along_axis(c.z - offset, c.ids.astype(np.int64), 1).astype(np.float32)
    c.t += np.random.default_rng(187).normal(0, 0.1, c.t.shape).astype(np.float32)
    c.dev = (c.dev[0], torch.from_numpy(c.t).cuda())
    say("distill offset", dtype, M, V, k, tau, offset)
    loss, d = c.run()
    alone = lpv.distill_loss(c.logits, *c.dev, tau)
    want = ft.distill(c.z, c.ids, c.t, tau)
    bound = np.zeros(M)
    for r in range(M):
        z, t = c.z[r] / tau, c.t[r].astype(np.float64) / tau
        dz, dt = z.max() - z, t.max() - t
        p = np.exp(-dz)
        lp = np.log(p.sum())
        q = np.exp(-dt)
        lq = np.log(q.sum())
        q /= q.sum()
        p /= p.sum()
        # the module's errors of a weight and of the two sums; a term of the cross sum holds
        # -dt - lq and d, and behind it log sum: off by 2^-22 of each, and of up to 2^-20 of them by
        # the sum over the entries (16 additions each)
        e_sum = (p * 2.0 ** -22 * (2 + 2 * dz)).sum() + 2.0 ** -16
        e_qs = (q * 2.0 ** -22 * (2 + 2 * dt)).sum() + 2.0 ** -18
        at = c.ids[r]
        size = dt + lq + dz[at] + lp
        term = np.abs(-dt - lq + dz[at] + lp)
        e = q * ((2.0 ** -22 * (2 + 2 * dt) + e_qs) * term + (2.0 ** -22 + 2.0 ** -20) * (size + 2))
        bound[r] = tau ** 2 * (e.sum() + e_qs + e_sum) + 2.0 ** -22 * abs(want[r])
    c.within(f64(loss), want, bound, "loss")
    c.within(f64(alone), want, bound, "loss alone")


@pytest.mark.parametrize("M,V", [(7, 1000), (7, 9000), (7, 120000)])
def test_a_diverged_row_does_not_read_as_zero(M, V):
    """A NaN among the student's logits, under one of the teacher's classes, beside them or
    everywhere, or among the teacher's: the loss is NaN, alone and with the gradient; rows without
    entries stay 0, and a class of the teacher's that the student leaves out is infinite."""
    def edit(c):
        c.z[0, c.ids[0, 2]] = np.nan
        c.z[1] = np.nan
        c.z[2, (c.ids[2].max() + 1) % V] = np.nan
        c.z[3, c.ids[3]] = -np.inf
        c.ids[4] = -1
        c.z[4, 5] = np.nan
        c.t[5, 3] = np.nan
        c.t[6] = np.nan
    c = Case(M, V, 12, "f32", seed=188, edit=edit)
    alone = lpv.distill_loss(c.logits, *c.dev, c.tau)
    loss, d = lpv.distill_grad(c.logits, *c.dev, c.tau, c.dloss)
    torch.cuda.synchronize()
    for x in (alone, loss):
        assert bool(torch.isnan(x[[0, 1, 2, 5, 6]]).all()) and x[3] == float("inf") and x[4] == 0
    assert not d[4].any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [1, 10, 1003, 21841])
def test_no_rows_of_any_number_of_classes(V, dtype):
    z = torch.empty((0, V), dtype=TORCH[dtype], device="cuda")
    ids, t = torch.empty((0, 3), dtype=torch.int32, device="cuda"), torch.empty((0, 3), device="cuda")
    assert lpv.distill_loss(z, ids, t, 1.0).shape == (0,)
    loss, d = lpv.distill_grad(z, ids, t, 1.0)
    assert loss.shape == (0,) and d.shape == (0, V)
    loss, d = lpv.distill_grad(z, ids, t, 1.0, dlogits=z)
    assert d is z
