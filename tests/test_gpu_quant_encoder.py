"""The encoder chain in 8 bits: every step against the oracle on its own input, graph replays
against the eager result, with and without a position bias."""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from oracle import encoder as enc
from oracle import quant
from gpu_util import assert_close, dev, f64, host, say
from test_gpu_quant_linear import check as check_linear
from test_gpu_quant_rows import check as check_rows
from test_gpu_quant_rows import sum_of

pytestmark = pytest.mark.gpu


def line_index(T):
    i = np.arange(T)
    return np.clip(i[None, :] - i[:, None], -8, 8).astype(np.int32) + 8


@pytest.mark.parametrize("n_seq,T,biased", [(2, 197, False), (3, 49, True)])
def test_encoder_chain_in_8_bits(n_seq, T, biased):
    from paper_2407_02068_amd import lpv
    from paper_2407_02068_amd.encoder import deit_chain
    H, blocks, eps = 12, 2, 1e-6
    layers = wl.b_stack(M=n_seq * T, layers=blocks)
    kw = {}
    if biased:
        tables = [dev(wl.quantize(wl.rng(126, i, 50).normal(0, 0.5, (17, H)).astype(np.float32), "bf16"), "bf16")
                  for i in range(blocks)]
        kw = {"relpos": lpv.relpos(torch.from_numpy(line_index(T)).cuda(), 17), "tables": tables}
    chain = deit_chain(layers, lambda a: dev(a, "bf16"), n_seq, T, H, eps, **kw)
    x0 = dev(layers[0].X, "bf16")
    with pytest.raises(ValueError):
        chain.run(x0, quant=True)
    chain.quantize()
    with pytest.raises(ValueError):
        chain.quantize()
    with pytest.raises(ValueError):
        chain.run(x0, sparse=False, quant=True)
    with pytest.raises(ValueError):
        chain.run(x0, quant=True, linear_events=[])
    weights, seen = {}, []
    for w in layers:
        W = oracle.decode(w.W, "bf16").reshape(w.W.shape)
        codes, scale = quant.codes(quant.keep(W, w.mask, w.b_r, w.b_c))
        weights[w.name] = w, codes, scale.astype(np.float32).astype(np.float64)
    g, b = np.ones(768), np.zeros(768)

    def trace(name, ins, out):
        torch.cuda.synchronize()
        seen.append(name)
        if name in weights:
            w, codes, scale = weights[name]
            bias = oracle.decode(w.bias, "bf16")
            ref = quant.linear(ins["q"].cpu().numpy(), f64(ins["scale"]), codes, scale, bias, w.gelu)
            check_linear(out, ref, "bf16", w.gelu, name)
        elif name.endswith("attention"):
            if not biased:
                x = oracle.decode(host(ins["qkv"], "bf16"), "bf16").reshape(n_seq * T, -1)
                assert_close(f64(out), enc.attention(x, n_seq, T, H, 64), "bf16", name)
        else:
            x, y = ins["x"], ins.get("y")
            s = f64(x) if y is None else f64(x) + f64(y)
            check_rows(out, quant.layer(s, g, b, eps) if "ln" in name else quant.codes(s), name)
            if ins.get("s") is not None:
                assert torch.equal(ins["s"], sum_of(x, y))

    x, A = chain.run(x0, trace=trace, quant=True)
    torch.cuda.synchronize()
    assert len(seen) == 1 + 9 * blocks - 1 and set(weights) < set(seen)
    ref = x.clone(), A.clone()
    x16, A16 = (t.clone() for t in chain.run(x0))
    say("  8 bits against 16: %.3g of the norm" % float((ref[1].float() - A16.float()).norm() / A16.float().norm()))
    assert torch.isfinite(ref[1].float()).all() and not torch.equal(A16, ref[1])
    graph, (xg, Ag) = chain.capture(x0, quant=True)
    for _ in range(3):
        chain.run(x0, sparse=False)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(xg, ref[0]) and torch.equal(Ag, ref[1])
    chain.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_root_mean_square_block_in_8_bits(dtype):
    """norm -> linear with GELU -> rows -> pruned linear -> the next norm, as one would chain them,
    each on what the one before it gave; float32 too."""
    from paper_2407_02068_amd import lpv
    from test_gpu_quant_linear import Case
    M, D, F = 131, 320, 1040
    up, down = Case(M, F, D, dtype), Case(M, D, F, dtype, 32, 16, 60)
    g = torch.Generator(device="cuda").manual_seed(3)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(up.bias.dtype)
    # (weights as a model has them: outputs of about 1, which float16 holds)
    up.W, up.ws = lpv.quant_rows(n(F, D) / D ** 0.5)
    down.W, down.ws = lpv.quant_rows(n(D, F) / F ** 0.5)
    hu, hd = up.pack(), down.pack()
    x, y, gamma = n(M, D), n(M, D), 1 + n(D) / 4
    S = torch.empty_like(x)
    for _ in range(2):
        ref = quant.rms(f64(x) + f64(y), f64(gamma), 1e-5)
        q, scale = lpv.add_rmsnorm_quant(x, y, gamma, 1e-5, S=S)
        check_rows((q, scale), ref, "norm")
        up.X, up.xs = q, scale
        z = lpv.quant_linear(hu, q, scale, up.bias, epi="gelu")
        check_linear(z, up.want(True), dtype, True, "up")
        q, scale = lpv.quant_rows(z)
        check_rows((q, scale), quant.codes(f64(z)), "rows")
        down.X, down.xs = q, scale
        y = lpv.quant_linear(hd, q, scale, down.bias)
        check_linear(y, down.want(), dtype, False, "down")
        x = S.clone()
