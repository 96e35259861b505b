"""Calls whose arrays have more than 2^31 elements, or more than 2^31 groups to convert: what they give at the far end is what the same rows give
alone, bit by bit (a row's arithmetic does not depend on where it lies)."""
import pytest
import torch

from paper_2308_14711_b200 import binding
from paper_2308_14711_b200.binding import FFFLayer

pytestmark = pytest.mark.gpu

FAR = 1 << 31


@pytest.fixture(autouse=True)
def room():
    yield
    torch.cuda.empty_cache()


def tree(depth):
    L = 1 << depth
    z = lambda *s: torch.zeros(s, device="cuda")
    return FFFLayer(1, 1, depth, 1, "relu", "f32", z(L - 1, 1), None, z(L, 1, 1), None, z(L, 1, 1), None)


@pytest.mark.parametrize("depth,B", [(8, 8_500_001), (15, 66_001)])
def test_routing_losses(depth, B):
    L, n = 1 << depth, 1000
    assert B * (L - 1) > FAR
    layer = tree(depth)
    g = torch.Generator("cuda").manual_seed(depth)
    mix = torch.rand(B, L, device="cuda", generator=g)
    leaf = torch.randint(0, L, (B,), device="cuda", generator=g, dtype=torch.int32)
    tail, last, one = mix[-n:].clone(), leaf[-n:].clone(), torch.ones(1, device="cuda")
    mask = torch.zeros(B, dtype=torch.bool, device="cuda")
    mask[-n:] = True
    loss, counts, mean = layer.balance_loss(mix, leaf, token_mask=mask)
    assert torch.equal(counts.long(), torch.bincount(last.long(), minlength=L))
    # n additions in float32 at most, 46 more in a CTA and one rounding, each 2^-24 of a mean that is not negative
    assert ((mean.double() - tail.double().mean(0)).abs() <= (n + 47) * 2.0 ** -24 * tail.double().mean(0)).all()
    dz = layer.routing_backward(mix, leaf_idx=leaf, counts=counts, dloss=one)
    assert torch.equal(dz[-n:], layer.routing_backward(tail, leaf_idx=last, counts=counts, dloss=one))
    del dz, mix
    dmix = layer.balance_loss_backward(leaf, counts, one)
    assert torch.equal(dmix[-n:], layer.balance_loss_backward(last, counts, one))
    layer.close()


@pytest.mark.parametrize("dtype,rows,cols", [(torch.bfloat16, 68_000, 32_000), (torch.bfloat16, 2_200_001, 1000), (torch.bfloat16, 2_200_001, 999),
                                             (torch.float32, 2_200_001, 999), (torch.bfloat16, 540_000_001, 1), (torch.float32, 540_000_001, 3)],
                         ids=["blocks", "groups", "any", "any_f32", "short_rows", "short_rows_f32"])
def test_conversion(dtype, rows, cols):
    nb = (cols + 31) // 32
    assert rows * cols > FAR or rows * nb * 4 > FAR
    n = 5000
    w = torch.empty(rows, cols, dtype=dtype, device="cuda")
    w[:rows // 2].fill_(3.0)
    w[rows // 2:].fill_(-1.5)
    w[-n:] = torch.randn(n, cols, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    codes, scales, values = binding.quantize_mx4(w, want_values=True)
    alone = binding.quantize_mx4(w[-n:].clone(), want_values=True)
    for got, want in zip((codes, scales, values), alone):
        assert torch.equal(got[-n:], want)
    assert (values[0] == 3.0).all() and (values[rows // 2 - 1] == 3.0).all() and (values[rows // 2] == -1.5).all()
    del w, values
    back = binding.dequantize_mx4(codes, scales, cols, dtype)
    assert torch.equal(back[-n:], alone[2]) and (back[0] == 3.0).all() and (back[rows // 2] == -1.5).all()


@pytest.mark.parametrize("D,O,depth,l,B", [(64, 2200, 4, 8, 1_000_000), (64, 1024, 4, 12, 2_200_000), (64, 1023, 4, 12, 2_200_000), (1023, 64, 3, 24, 2_200_000),
                                           (64, 1023, 4, 3, 2_200_000)], ids=["lists", "out", "odd_out", "odd_in", "thin"])
def test_4_bit_layers(D, O, depth, l, B):
    assert B * max(D, O) > FAR
    n, leaves = 5000, 1 << depth
    g = torch.Generator("cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.bfloat16)
    layer = FFFLayer.from_mx4(D, O, depth, l, "gelu", rnd(leaves - 1, D), rnd(leaves - 1), *binding.quantize_mx4(rnd(leaves, l, D)), rnd(leaves, l),
                              *binding.quantize_mx4(rnd(leaves, l, O)), rnd(leaves, O))
    x = rnd(B, D)
    y, leaf = layer.forward_infer(x)
    torch.cuda.synchronize()
    assert layer.last_status() == 0
    tail, last = layer.forward_infer(x[-n:].clone())
    assert torch.equal(leaf[-n:], last) and torch.equal(y[-n:], tail)
    del y
    layer.close()
