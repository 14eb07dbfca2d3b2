"""What the 8-bit calls promise beside their results: the accuracy of the GELU of float32 outputs on the device,
no allocation, and the position-biased attention of a chain in 8 bits."""
import numpy as np
import pytest
import torch
from scipy.special import erfc

import oracle
import workloads as wl
from gpu_util import dev, f64, host, kernels, say
from test_gpu_finetune import Attention, window_index

pytestmark = pytest.mark.gpu


def lpv():
    from paper_2407_02068_amd import lpv as m
    m.lib()
    return m


@pytest.mark.parametrize("M,N,K,kernel", [
    (1, 44800, 16, "few<0, true, 4, 4>"), (1, 4096, 2048, "few<0, true, 8, 4>"), (150, 16384, 16, "panel<0, true, 1, 4, 4>"),
    (150, 65536, 16, "panel<0, true, 2, 4, 4>"), (1024, 16384, 2048, "panel<0, true, 4, 8, 4>")])
def test_gelu_of_float32_outputs(M, N, K, kernel):
    """Sums of 0 leave the bias alone, which sweeps -8 to 12.  The formula step by step in float32 is within
    1.74e-7 of positive outputs (relative) and 4.4e-8 of negative ones, past the cut at -5.66 too; the
    exponential's instruction adds one unit in the last place of its term, 2^-23 of at most the output
    (|v| / 2 where v is small) and of at most 0.17: 2.93e-7 and 6.5e-8, inside the stated 3e-7 and 1e-7."""
    m = lpv()
    v = torch.linspace(-8, 12, N, device="cuda")
    v = torch.where(v == 0, 0.5, v).contiguous()
    h = m.quant_pack(torch.ones((N, K), dtype=torch.int8, device="cuda"), torch.ones(N, device="cuda"))
    X, xs = torch.zeros((M, K), dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda")
    Y = m.quant_linear(h, X, xs, v, epi="gelu")
    assert kernels(lambda: m.quant_linear(h, X, xs, v, epi="gelu"), args=True) == {"k_quant_" + kernel}
    assert torch.equal(Y, Y[:1].expand_as(Y))
    x = f64(v)
    ref = x * 0.5 * erfc(-x / np.sqrt(2.0))
    err = np.abs(f64(Y[0]) - ref)
    up = x > 0
    say("  %s: %.3g of positive outputs, %.3g of negative ones" % (kernel, (err[up] / ref[up]).max(), err[~up].max()))
    assert (err[up] <= 3e-7 * ref[up]).all() and (err[~up] <= 1e-7).all()


@pytest.mark.parametrize("M,N,K", [(1, 96, 64), (300, 1040, 80), (4000, 2064, 2064)])
def test_no_allocation(M, N, K, monkeypatch):
    # (the library's own allocations fail: packing does, and no other call notices)
    m = lpv()
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16)
    one = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    W, ws = m.quant_rows(torch.randn((N, K), generator=g, device="cuda").to(torch.bfloat16))
    h = m.quant_pack(W, ws)
    q, scale = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    Y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")

    def run():
        outs = []
        for call in (lambda: m.quant_rows(x, x, q=q, scale=scale), lambda: m.add_rmsnorm_quant(x, x, one, 1e-6, q=q, scale=scale),
                     lambda: m.add_layernorm_quant(x, x, one, one, 1e-6, q=q, scale=scale)):
            call()
            outs += [q.clone(), scale.clone()]
            m.quant_linear(h, q, scale, Y=Y, epi="gelu")
            outs.append(Y.clone())
        return outs

    want = run()
    monkeypatch.setenv("LPV_FAULT_INJECT", "alloc")
    with pytest.raises(m.LpvError, match="LPV_ERR_ALLOC"):
        m.quant_pack(W, ws)
    assert all(torch.equal(a, b) for a, b in zip(run(), want))


@pytest.mark.parametrize("labels", [False, True])
def test_the_biased_attention_of_a_chain_in_8_bits(labels):
    """On its own input, against the oracle and the call itself."""
    from paper_2407_02068_amd.encoder import deit_chain
    m = lpv()
    H, blocks, n_seq = 12, 2, 3
    idx, n = window_index(7, False)
    T = len(idx)
    layers = wl.b_stack(M=n_seq * T, layers=blocks)
    region = None
    if labels:
        region = np.zeros((1, T), np.int32)
        region[0, T // 3:] = 1
        region[0, -5:] = -1
    bits = [wl.quantize(wl.rng(127, i, 50).normal(0, 0.5, (n, H)).astype(np.float32), "bf16") for i in range(blocks)]
    tables = [dev(b, "bf16") for b in bits]
    rp = m.relpos(torch.from_numpy(idx).cuda(), n)
    reg = None if region is None else torch.from_numpy(region).cuda()
    chain = deit_chain(layers, lambda a: dev(a, "bf16"), n_seq, T, H, relpos=rp, tables=tables, region=reg)
    chain.quantize()
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

        c = Attention(idx, n, n_seq, H, 64, "bf16", region=region, edit=edit)
        lse = torch.empty((n_seq, H, T), device="cuda")
        assert torch.equal(m.relpos_attention(rp, tables[blk], ins["qkv"], n_seq, H, region=reg, lse=lse), out)
        c.check(out, lse)
        seen.append(blk)

    chain.run(dev(layers[0].X, "bf16"), trace=trace, quant=True)
    assert seen == [0, 1]
    chain.close()
