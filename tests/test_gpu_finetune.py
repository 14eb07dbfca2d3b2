"""GPU parity of the operators of finetuning as they are used together: a step of a pruned
block with position-biased attention, its head distilled from a teacher's top logits, back to
every parameter, and the encoder chain with a position bias.  Each link is checked against
the float64 oracle fed the GPU's own inputs of that link."""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from gpu_util import TOL, TORCH, dev, f64, host, say
from oracle import finetune as ft
from paper_2407_02068_amd import lpv
from paper_2407_02068_amd.encoder import EncoderChain, deit_chain
from test_gpu_distill import Case as Loss
from test_gpu_relpos import Case as Attention
from test_gpu_relpos import line_index, window_index

pytestmark = pytest.mark.gpu


def close(y, r, dtype, what, tile=32):
    """gpu_util's bar on every tile of the result, to which fp16 adds half its smallest step:
    the step's gradients reach its subnormal numbers (a value of 2^-17 is a whole number of
    2^-24 and rounds by up to 2^-25, 2^-8 of it, above the bar), so no multiple of the value
    bounds their rounding."""
    y, r = np.atleast_2d(y), np.atleast_2d(r)
    if r.ndim == 3:
        y, r = y.reshape(-1, r.shape[-1]), r.reshape(-1, r.shape[-1])
    worst = 0.0
    for i in range(0, r.shape[0], tile):
        for j in range(0, r.shape[1], tile):
            a, b = y[i:i + tile, j:j + tile], r[i:i + tile, j:j + tile]
            bound = TOL[dtype] * np.abs(b).max() + (2.0 ** -25 if dtype == "f16" else 0.0)
            worst = max(worst, float(np.abs(a - b).max() / (bound + 1e-300)))
    say("  %s: at most %.2f of its bound" % (what, worst))
    assert worst <= 1.0, "%s: %.3g times its bound" % (what, worst)


class Layer:
    """A packed linear layer, its transpose, and its parameters on the host."""

    def __init__(self, cfg, M, N, K, dtype, kind="uniform"):
        self.w = w = wl.custom(cfg, M, N, K, 16, 16, dtype, kind, 50)
        self.h = lpv.bsr_pack(dev(w.W, dtype), dev(w.mask), 16, 16)
        self.ht = lpv.bsr_transpose(self.h)
        self.b = dev(w.bias, dtype)

    def check(self, dtype, x, y, g, dx, dw, db, what):
        w = self.w
        x, g = host(x, dtype), host(g, dtype)
        close(f64(y), oracle.linear(x, w.W, dtype, 16, 16, w.mask, w.bias), dtype, what)
        close(f64(dx), oracle.grad_x(g, w.W, dtype, 16, 16, w.mask), dtype, what + " dX")
        close(f64(dw), oracle.grad_w(g, x, dtype, 16, 16, w.mask), dtype, what + " dW", tile=16)
        close(f64(db), oracle.grad_bias(g, dtype), dtype, what + " db")

    def close(self):
        self.h.close()
        self.ht.close()


class Step:
    """Forward, loss and backward of qkv -> attention -> proj -> head, for every token."""

    def __init__(self, idx, n_buckets, n_seq, H, V, k, dtype, region=None):
        self.dtype, self.n_seq, self.H, self.V, self.idx, self.region = dtype, n_seq, H, V, idx, region
        D, M, Vp = H * 32, n_seq * idx.shape[0], (V + 15) // 16 * 16
        self.qkv = Layer(121, M, 3 * D, D, dtype)
        self.proj = Layer(122, M, D, D, dtype, "bernoulli")
        self.head = Layer(123, M, Vp, D, dtype, "all")
        self.x = dev(self.qkv.w.X, dtype)
        r = wl.rng(124, 0, 50)
        self.table_bits = wl.quantize(r.normal(0, 0.5, (n_buckets, H)).astype(np.float32), dtype)
        self.table = dev(self.table_bits, dtype)
        self.rp = lpv.relpos(torch.from_numpy(idx).cuda(), n_buckets)
        self.reg = None if region is None else torch.from_numpy(region).cuda()
        self.ids = r.integers(0, V, (M, k)).astype(np.int32)
        self.ids[np.arange(k)[None, :] >= r.integers(0, k + 1, (M, 1))] = -1  # (0 to k entries)
        self.t = (8 - np.cumsum(r.exponential(0.4, (M, k)), 1)).astype(np.float32)
        self.g = np.full(M, 1.0 / 16, np.float32)
        self.teacher = (torch.from_numpy(self.ids).cuda(), torch.from_numpy(self.t).cuda())
        self.dloss = torch.from_numpy(self.g).cuda()
        self.lse = torch.empty((n_seq, H, idx.shape[0]), device="cuda")
        self.M, self.D, self.Vp, self.tau = M, D, Vp, 2.0

    def run(self):
        n, H = self.n_seq, self.H
        new = lambda rows, cols: torch.empty((rows, cols), dtype=TORCH[self.dtype], device="cuda")
        s = {"qkv": lpv.bsr_linear(self.qkv.h, self.x, self.qkv.b)}
        s["o"] = lpv.relpos_attention(self.rp, self.table, s["qkv"], n, H, region=self.reg,
                                      lse=self.lse, hd=32)
        s["p"] = lpv.bsr_linear(self.proj.h, s["o"], self.proj.b)
        s["z"] = lpv.bsr_linear(self.head.h, s["p"], self.head.b)
        s["dz"] = new(self.M, self.Vp)
        s["loss"], _ = lpv.distill_grad(s["z"][:, :self.V], *self.teacher, self.tau, self.dloss,
                                        dlogits=s["dz"])

        def back(layer, name, g, x):
            s["dw_" + name] = lpv.grad_w(layer.h, g, x)
            s["db_" + name] = lpv.bias_grad_noalloc(g, new(1, g.shape[1])[0])
            return lpv.bsr_linear(layer.ht, g)
        s["dp"] = back(self.head, "head", s["dz"], s["p"])
        s["do"] = back(self.proj, "proj", s["dp"], s["o"])
        s["dqkv"], s["dtable"] = lpv.relpos_attention_grad(self.rp, self.table, s["qkv"], s["o"], self.lse,
                                                           s["do"], n, H, region=self.reg, hd=32)
        s["dx"] = back(self.qkv, "qkv", s["dqkv"], self.x)
        s["lse"] = self.lse
        return s

    def check(self, s):
        dt = self.dtype
        dec = lambda t: oracle.decode(host(t, dt), dt).reshape(t.shape)
        self.qkv.check(dt, self.x, s["qkv"], s["dqkv"], s["dx"], s["dw_qkv"], s["db_qkv"], "qkv")
        self.proj.check(dt, s["o"], s["p"], s["dp"], s["do"], s["dw_proj"], s["db_proj"], "proj")
        self.head.check(dt, s["p"], s["z"], s["dz"], s["dp"], s["dw_head"], s["db_head"], "head")

        def attention(c):
            c.x, c.t, c.g = dec(s["qkv"]), oracle.decode(self.table_bits, dt).reshape(self.table.shape), dec(s["do"])
        c = Attention(self.idx, self.rp.n_buckets, self.n_seq, self.H, 32, dt, region=self.region,
                      edit=attention)
        c.check(s["o"], s["lse"], s["dqkv"], s["dtable"])

        def loss(c):
            c.z, c.ids, c.t, c.g = dec(s["z"])[:, :self.V], self.ids, self.t, self.g
        c = Loss(self.M, self.V, self.ids.shape[1], dt, tau=self.tau, edit=loss)
        c.check(s["loss"], s["dz"][:, :self.V])
        assert not s["dz"][:, self.V:].any()

    def close(self):
        for layer in (self.qkv, self.proj, self.head):
            layer.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["window", "line", "long"])
def test_finetuning_step(kind, dtype):
    say("finetuning step", kind, dtype)
    region = None
    if kind == "window":
        idx, n = window_index(7)
        region = np.random.default_rng(7).integers(0, 2, (3, 49)).astype(np.int32)
        region[2, 30:] = -1
    else:
        idx, n = line_index(75 if kind == "line" else 230)
    s = Step(idx, n, 6 if kind == "window" else 2, 3, 1003, 9, dtype, region)
    s.check(s.run())
    torch.cuda.synchronize()
    s.close()


def test_finetuning_step_captured():
    """The step in a graph: replays between eager steps, and after the results were
    overwritten, give the eager step's bits; a second graph of the same step does too."""
    say("finetuning step, captured")
    idx, n = window_index(7)
    s = Step(idx, n, 20, 3, 100, 7, "bf16")
    ref = {k: v.clone() for k, v in s.run().items()}
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = s.run()
        graphs.append((graph, out))
    for i in range(3):
        s.run()
        for graph, out in graphs:
            for v in out.values():
                v.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for k, v in out.items():
                assert torch.equal(v, ref[k]), (i, k)
    s.close()


@pytest.mark.parametrize("side,class_token,n_seq,labels", [(14, True, 2, False), (14, True, 2, True),
                                                           (7, False, 5, True)])
def test_encoder_chain_with_a_position_bias(side, class_token, n_seq, labels):
    """Every attention of the chain against the oracle on its own input, and graph replays."""
    H, blocks = 12, 2
    idx, n = window_index(side, class_token)
    T = len(idx)
    layers = wl.b_stack(M=n_seq * T, layers=blocks)
    region = None
    if labels:
        region = np.zeros((1, T), np.int32)
        region[0, T // 3:] = 1
        region[0, -5:] = -1
    bits = [wl.quantize(wl.rng(125, i, 50).normal(0, 0.5, (n, H)).astype(np.float32), "bf16")
            for i in range(blocks)]
    tables = [dev(b, "bf16") for b in bits]
    rp = lpv.relpos(torch.from_numpy(idx).cuda(), n)
    reg = None if region is None else torch.from_numpy(region).cuda()
    chain = deit_chain(layers, lambda a: dev(a, "bf16"), n_seq, T, H, relpos=rp, tables=tables, region=reg)
    seen = []

    def trace(name, ins, out):
        if name.endswith("attention"):
            torch.cuda.synchronize()
            blk = int(name.split(".")[0])
            x = oracle.decode(host(ins["qkv"], "bf16"), "bf16").reshape(n_seq * T, -1)
            t = oracle.decode(bits[blk], "bf16").reshape(n, H)

            def edit(c):
                c.x, c.t = x, t

            c = Attention(idx, n, n_seq, H, 64, "bf16", region=region, edit=edit)
            lse = torch.empty((n_seq, H, T), device="cuda")
            again = lpv.relpos_attention(rp, tables[blk], ins["qkv"], n_seq, H, region=reg, lse=lse)
            assert torch.equal(again, out)
            c.check(out, lse)
            seen.append(blk)
    x0 = dev(layers[0].X, "bf16")
    x, A = chain.run(x0, trace=trace)
    torch.cuda.synchronize()
    assert seen == [0, 1]
    ref = x.clone(), A.clone()
    graph, (xg, Ag) = chain.capture(x0)
    for _ in range(3):
        chain.run(x0, sparse=False)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(xg, ref[0]) and torch.equal(Ag, ref[1])
    for kw in ({"tables": tables}, {"relpos": rp}, {"relpos": rp, "tables": tables[:1]}, {"region": x0}):
        with pytest.raises(ValueError):
            EncoderChain(chain.linears, n_seq, T, H, chain.gamma, chain.beta, **kw)
    with pytest.raises(ValueError):
        EncoderChain(chain.linears, n_seq, T - 1, H, chain.gamma, chain.beta, relpos=rp, tables=tables)
    chain.close()


def check_chain(H, regions, region):
    """A chain of 768 / H dimensions to a head: every attention against the oracle on its own input
    and its block's labels, and graph replays."""
    n_seq, T, blocks, hd = 2, 40, len(regions), 768 // H
    idx, n = line_index(T, 16)
    layers = wl.b_stack(M=n_seq * T, layers=blocks)
    bits = [wl.quantize(wl.rng(126, i, 50).normal(0, 0.5, (n, H)).astype(np.float32), "bf16")
            for i in range(blocks)]
    tables = [dev(b, "bf16") for b in bits]
    rp = lpv.relpos(torch.from_numpy(idx).cuda(), n)
    chain = deit_chain(layers, lambda a: dev(a, "bf16"), n_seq, T, H, relpos=rp, tables=tables, region=region)
    seen = []

    def trace(name, ins, out):
        if not name.endswith("attention"):
            return
        torch.cuda.synchronize()
        blk = int(name.split(".")[0])
        x = oracle.decode(host(ins["qkv"], "bf16"), "bf16").reshape(n_seq * T, -1)
        t = oracle.decode(bits[blk], "bf16").reshape(n, H)

        def edit(c):
            c.x, c.t = x, t

        c = Attention(idx, n, n_seq, H, hd, "bf16", region=regions[blk], edit=edit)
        lse = torch.empty((n_seq, H, T), device="cuda")
        again = lpv.relpos_attention(rp, tables[blk], ins["qkv"], n_seq, H, region=c.reg, lse=lse, hd=hd)
        assert torch.equal(again, out)
        c.check(out, lse)
        seen.append(blk)
    x0 = dev(layers[0].X, "bf16")
    x, A = chain.run(x0, trace=trace)
    torch.cuda.synchronize()
    assert seen == list(range(blocks))
    ref = x.clone(), A.clone()
    graph, (xg, Ag) = chain.capture(x0)
    for _ in range(3):
        chain.run(x0, sparse=False)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(xg, ref[0]) and torch.equal(Ag, ref[1])
    return chain, rp, tables


@pytest.mark.parametrize("H", [12, 24])
def test_encoder_chain_of_other_heads(H):
    """The position bias with heads of 64 and of 32 dimensions."""
    say("encoder chain", H, "heads")
    check_chain(H, [None, None], None)[0].close()


def test_encoder_chain_with_labels_by_block():
    """The plain and the shifted windows of a row of tokens in turn, and all tokens in a block without
    labels."""
    at = np.arange(40)
    regions = [(at // 8)[None], None, np.stack([(at + 4) // 8, np.where(at < 30, (at + 4) // 8, -1)])]
    regs = [None if r is None else torch.from_numpy(r.astype(np.int32)).cuda() for r in regions]
    say("encoder chain, labels by block")
    chain, rp, tables = check_chain(24, regions, regs)
    for bad in (regs[:2], regs + [None], []):
        with pytest.raises(ValueError):
            EncoderChain(chain.linears, 2, 40, 24, chain.gamma, chain.beta, relpos=rp, tables=tables, region=bad)
    chain.close()
