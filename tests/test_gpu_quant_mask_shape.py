"""The block mask of a weight in 8-bit codes: its shape."""
import pytest
import torch

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
