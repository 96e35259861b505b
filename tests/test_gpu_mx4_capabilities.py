"""What fff_capabilities says of 4-bit layers: the bits of tensor-core kernels promise rows taken as they are."""
import pytest
import torch

from paper_2308_14711_b200 import binding
from paper_2308_14711_b200.binding import FFFLayer

pytestmark = pytest.mark.gpu

DESCENT, TCGEN05, LEAF, PADDED = 1, 2, 4, 128


@pytest.mark.parametrize("D,O,l,has", [
    (1024, 64, 12, DESCENT | TCGEN05 | LEAF), (1024, 64, 7, DESCENT | TCGEN05), (1024, 61, 12, DESCENT | TCGEN05),
    (1023, 64, 12, PADDED), (1017, 64, 12, PADDED), (1023, 64, 7, PADDED), (1000, 64, 12, PADDED), (1016, 61, 12, PADDED), (121, 8, 8, PADDED),
])
def test_capabilities(D, O, l, has):
    depth, n = 6, 64
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
    layer = FFFLayer.from_mx4(D, O, depth, l, "gelu", rnd(n - 1, D), rnd(n - 1), *binding.quantize_mx4(rnd(n, l, D)),
                              rnd(n, l), *binding.quantize_mx4(rnd(n, l, O)), rnd(n, O))
    assert layer.capabilities() & (DESCENT | TCGEN05 | LEAF | 8 | PADDED) == has
    layer.close()
