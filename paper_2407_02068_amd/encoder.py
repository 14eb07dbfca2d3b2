"""The DeiT encoder with the pruned linear layers in place, chained on the GPU.

Composition only: every step is one liblpv call (lpv.py), nothing is computed
here.  The paper prunes the four linear layers of every DeiT encoder block
(qkv, proj, fc1, fc2; Sec. 4) and compares whole-model inference (Tab. 2);
this chains the standard pre-norm block around them:

    A = LN(x)
    per block:  qkv = A Wqkv~^T + b         (block-sparse or dense)
                O   = attention(qkv)         (H heads of 64)
                P   = O Wproj~^T + b
                x   = x + P;  A = LN(x)
                Hd  = GELU(A Wfc1~^T + b)
                P   = Hd Wfc2~^T + b
                x   = x + P;  A = LN(x)      (the next block's first LN)

With a position bias (one table of buckets per block) the attention is the
position-biased one, in windows or over regions of tokens if labels are given.
In 8 bits (``quantize``, then ``run(..., quant=True)``) every linear layer takes 8-bit
codes with a scale for each token, from its own weight in 8-bit codes: the layer norms
give them in place of A, and O and Hd are quantised row by row.

Every layer norm uses the same gamma / beta.  The residual stream alternates
between two buffers, so a run never overwrites its own input and every run
computes the same function of ``x0``.
"""
import torch

from . import lpv


class Linear:
    """One linear layer of the chain on the device: the dense weight, its
    packed block-sparse handle (None until packed), bias and epilogue."""

    def __init__(self, name, W, mask, bias, b_r, b_c, gelu):
        self.name, self.W, self.mask, self.bias = name, W, mask, bias
        self.b_r, self.b_c, self.gelu = b_r, b_c, gelu
        self.h = lpv.bsr_pack(W, mask, b_r, b_c)
        self.q = None

    def quantize(self):
        """Packs the kept blocks in 8-bit codes with a scale for each output."""
        N, K = self.W.shape
        mask = self.mask.view(N // self.b_r, K // self.b_c)  # (bsr_pack takes its entries in any shape)
        keep = mask.repeat_interleave(self.b_r, 0).repeat_interleave(self.b_c, 1) != 0
        codes, scale = lpv.quant_rows(torch.where(keep, self.W, 0))
        self.q = lpv.quant_pack(codes, scale, mask, self.b_r, self.b_c)

    def __call__(self, x, y, sparse):
        epi = "gelu" if self.gelu else None
        if sparse:
            return lpv.bsr_linear(self.h, x, self.bias, y, epi=epi)
        return lpv.dense_linear(self.W, x, self.bias, y, epi=epi)

    def quant(self, codes, scale, y):
        return lpv.quant_linear(self.q, codes, scale, self.bias, y, epi="gelu" if self.gelu else None)

    def close(self):
        self.h.close()
        if self.q is not None:
            self.q.close()


class EncoderChain:
    """``blocks`` DeiT encoder blocks over M = n_seq * T tokens of width D.

    linears: 4 * blocks Linear objects in the order (qkv, proj, fc1, fc2) per
    block; gamma, beta: the layer norms' D-element parameters.  relpos (a
    lpv.RelPos of T tokens) with tables (one n_buckets x H table per block):
    attention with that position bias, heads of D / H = 32 or 64 dimensions (64
    without); region: its labels, as lpv.relpos_attention takes them, or a list
    of them, one for each block (None: a block without), as plain and shifted
    windows alternate."""

    def __init__(self, linears, n_seq, T, H, gamma, beta, eps=1e-6, relpos=None, tables=None,
                 region=None):
        if len(linears) % 4:
            raise ValueError("four linear layers per block")
        if relpos is None and (tables is not None or region is not None):
            raise ValueError("tables and region need relpos")
        if relpos is not None and (relpos.T != T or tables is None
                                   or len(tables) * 4 != len(linears)):
            raise ValueError("relpos of T tokens, with one table per block")
        if isinstance(region, (list, tuple)) and len(region) * 4 != len(linears):
            raise ValueError("one region for all blocks, or one for each")
        self.linears, self.n_seq, self.T, self.H = linears, n_seq, T, H
        self.gamma, self.beta, self.eps = gamma, beta, eps
        D = linears[0].W.shape[1]
        M = n_seq * T
        dt, dv = gamma.dtype, gamma.device
        new = lambda cols: torch.empty((M, cols), dtype=dt, device=dv)
        self.D, self.M = D, M
        self.A, self.O, self.P = new(D), new(D), new(D)
        self.qkv, self.Hd = new(linears[0].W.shape[0]), new(linears[2].W.shape[0])
        self.R = [new(D), new(D)]
        self.codes = None
        self.relpos, self.tables, self.region = relpos, tables, region
        self.relpos_ws = None
        if relpos is not None:
            self.relpos_ws = torch.empty(lpv.relpos_workspace_size(relpos, n_seq, H),
                                         dtype=torch.uint8, device=dv)

    @property
    def blocks(self):
        return len(self.linears) // 4

    def quantize(self):
        """Gets the chain ready for ``run(..., quant=True)``: every linear layer's weight in 8-bit
        codes, and the buffers of the activations' codes and scales.  Once only: captured
        graphs hold their addresses."""
        if self.codes is not None:
            raise ValueError("the chain is in 8 bits already")
        new = lambda cols: (torch.empty((self.M, cols), dtype=torch.int8, device=self.A.device),
                            torch.empty(self.M, dtype=torch.float32, device=self.A.device))
        for layer in self.linears:
            layer.quantize()
        self.codes = {"A": new(self.D), "O": new(self.D), "Hd": new(self.Hd.shape[1])}

    def _attention(self, blk, qkv, out):
        if self.relpos is None:
            return lpv.attention(qkv, self.n_seq, self.T, self.H, out=out)
        region = self.region[blk] if isinstance(self.region, (list, tuple)) else self.region
        return lpv.relpos_attention(self.relpos, self.tables[blk], qkv, self.n_seq, self.H,
                                    region=region, out=out, workspace=self.relpos_ws,
                                    hd=self.D // self.H)

    def _run_quant(self, x0, trace=None):
        """``run`` with 8-bit codes into every linear layer.  trace: as there; the codes and scales of
        a layer's input are its "q" and "scale"."""
        if self.codes is None:
            raise ValueError("quantize() first")
        g, b, eps = self.gamma, self.beta, self.eps
        O, P, qkv, Hd, R = self.O, self.P, self.qkv, self.Hd, self.R
        A8, O8, Hd8 = self.codes["A"], self.codes["O"], self.codes["Hd"]

        def lin(layer, x8, y):
            layer.quant(*x8, y)
            if trace:
                trace(layer.name, {"q": x8[0], "scale": x8[1]}, y)

        def norm(name, x, y, S):
            lpv.add_layernorm_quant(x, y, g, b, eps, S=S, q=A8[0], scale=A8[1])
            if trace:
                trace(name, {"x": x, "y": y, "s": S}, A8)

        def rows(name, x, x8):
            lpv.quant_rows(x, q=x8[0], scale=x8[1])
            if trace:
                trace(name, {"x": x}, x8)

        x, nxt = x0, 0
        norm("ln.in", x, None, None)
        for blk in range(self.blocks):
            q, pr, f1, f2 = self.linears[4 * blk:4 * blk + 4]
            lin(q, A8, qkv)
            self._attention(blk, qkv, O)
            if trace:
                trace("%d.attention" % blk, {"qkv": qkv}, O)
            rows("%d.o" % blk, O, O8)
            lin(pr, O8, P)
            norm("%d.add_ln1" % blk, x, P, R[nxt])
            x, nxt = R[nxt], 1 - nxt
            lin(f1, A8, Hd)
            rows("%d.hd" % blk, Hd, Hd8)
            lin(f2, Hd8, P)
            if blk + 1 < self.blocks:
                norm("%d.add_ln2" % blk, x, P, R[nxt])
            else:  # (the result: no layer takes it)
                lpv.add_layernorm(x, P, g, b, eps, S=R[nxt], out=self.A)
            x, nxt = R[nxt], 1 - nxt
        return x, self.A

    def run(self, x0, sparse=True, trace=None, linear_events=None, quant=False):
        """One forward pass from the token activations x0 (M x D).  Returns
        (x, A): the residual stream after the last block and its layer norm.
        quant: every linear layer in 8 bits, over its kept blocks (after ``quantize``; it takes
        neither sparse=False nor linear_events).

        trace(name, inputs, output), if given, is called after every step with
        the step's input tensors (a dict) and its output, for checking a link
        at a time.  linear_events, if a list, receives a (start, end) pair of
        timing events recorded around every linear launch."""
        if quant:
            if not sparse or linear_events is not None:
                raise ValueError("in 8 bits the chain is sparse, and records no events")
            return self._run_quant(x0, trace)
        g, b, eps = self.gamma, self.beta, self.eps
        A, O, P, qkv, Hd, R = self.A, self.O, self.P, self.qkv, self.Hd, self.R

        def lin(layer, x, y):
            if linear_events is not None:
                e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                e0.record()
                layer(x, y, sparse)
                e1.record()
                linear_events.append((e0, e1))
            else:
                layer(x, y, sparse)
            if trace:
                trace(layer.name, {"x": x}, y)

        x, nxt = x0, 0
        lpv.add_layernorm(x, None, g, b, eps, out=A)
        if trace:
            trace("ln.in", {"x": x}, A)
        for blk in range(self.blocks):
            q, pr, f1, f2 = self.linears[4 * blk:4 * blk + 4]
            lin(q, A, qkv)
            self._attention(blk, qkv, O)
            if trace:
                trace("%d.attention" % blk, {"qkv": qkv}, O)
            lin(pr, O, P)
            lpv.add_layernorm(x, P, g, b, eps, S=R[nxt], out=A)
            if trace:
                trace("%d.add_ln1" % blk, {"x": x, "y": P, "s": R[nxt]}, A)
            x, nxt = R[nxt], 1 - nxt
            lin(f1, A, Hd)
            lin(f2, Hd, P)
            lpv.add_layernorm(x, P, g, b, eps, S=R[nxt], out=A)
            if trace:
                trace("%d.add_ln2" % blk, {"x": x, "y": P, "s": R[nxt]}, A)
            x, nxt = R[nxt], 1 - nxt
        return x, A

    def capture(self, x0, sparse=True, quant=False):
        """The forward pass from x0 captured once into a HIP graph (through
        torch.cuda.CUDAGraph): replaying it relaunches the same 1 + 7 * blocks (in 8
        bits 1 + 9 * blocks) calls' kernels on the same buffers with no host work per launch.  Every call
        of the chain is capturable (no allocation, no host synchronisation, no
        memset); one eager pass first settles the kernels' one-time set-up.
        Returns (graph, (x, A)): the outputs the replays rewrite."""
        self.run(x0, sparse, quant=quant)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = self.run(x0, sparse, quant=quant)
        torch.cuda.synchronize()
        return graph, out

    def close(self):
        for layer in self.linears:
            layer.close()


def deit_chain(layers, to_dev, n_seq, T=197, H=12, eps=1e-6, relpos=None, tables=None,
               region=None):
    """An EncoderChain from generated layer inputs (objects with W, mask, bias,
    b_r, b_c, gelu, name as numpy arrays; ``to_dev`` moves an array of the
    element type to the GPU).  Layer norms: gamma = 1, beta = 0.
    relpos, tables, region: as EncoderChain takes them."""
    lins = [Linear(w.name, to_dev(w.W), torch.from_numpy(w.mask).cuda(), to_dev(w.bias),
                   w.b_r, w.b_c, w.gelu) for w in layers]
    D = lins[0].W.shape[1]
    dt = lins[0].W.dtype
    gamma = torch.ones(D, dtype=dt, device="cuda")
    beta = torch.zeros(D, dtype=dt, device="cuda")
    return EncoderChain(lins, n_seq, T, H, gamma, beta, eps, relpos, tables, region)
