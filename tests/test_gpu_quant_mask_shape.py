"""The block mask of a weight in 8-bit codes: its shape, and a flat one through the encoder chain."""
import pytest
import torch

import workloads as wl
from gpu_util import dev

pytestmark = pytest.mark.gpu


def lpv():
    from paper_2407_02068_amd import lpv as m
    m.lib()
    return m


def test_a_mask_of_another_shape_is_refused():
    # as many entries, in other rows: the blocks that it keeps would be others
    m = lpv()
    g = torch.Generator(device="cuda").manual_seed(1)
    W = torch.randint(-128, 128, (64, 96), generator=g, device="cuda").to(torch.int8)
    ws, xs = torch.rand(64, generator=g, device="cuda"), torch.rand(5, generator=g, device="cuda")
    X = torch.randint(-128, 128, (5, 96), generator=g, device="cuda").to(torch.int8)
    mask = torch.randint(0, 2, (4, 3), generator=g, device="cuda").to(torch.uint8)
    for other in (mask.t().contiguous(), mask.view(2, 6), mask.view(12, 1), mask.view(1, 4, 3), mask[:, :2].contiguous(),
                  mask.view(-1)[:11]):
        with pytest.raises(ValueError, match="mask"):
            m.quant_pack(W, ws, other, 16, 32)
    want = m.quant_linear(m.quant_pack(W, ws, mask, 16, 32), X, xs)
    flat = m.quant_linear(m.quant_pack(W, ws, mask.view(-1), 16, 32), X, xs)  # (row by row)
    assert torch.equal(want, flat)


def test_a_chain_of_flat_masks():
    # the 16-bit chain takes them; so does the one in 8 bits
    from paper_2407_02068_amd.encoder import EncoderChain, Linear
    n_seq, T, H = 1, 50, 12
    layers = wl.b_stack(M=n_seq * T, layers=1)
    outs = []
    for flat in (False, True):
        lins = []
        for w in layers:
            mask = dev(w.mask)
            lins.append(Linear(w.name, dev(w.W, "bf16"), mask.view(-1) if flat else mask, dev(w.bias, "bf16"),
                               w.b_r, w.b_c, w.gelu))
        one = torch.ones(768, dtype=torch.bfloat16, device="cuda")
        chain = EncoderChain(lins, n_seq, T, H, one, torch.zeros_like(one))
        x0 = dev(layers[0].X, "bf16")
        a = [t.clone() for t in chain.run(x0)]
        chain.quantize()
        outs.append(a + [t.clone() for t in chain.run(x0, quant=True)])
        chain.close()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
