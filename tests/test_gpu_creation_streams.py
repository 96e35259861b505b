"""Layers and stacks made on a stream that does not wait for the default one, right behind the work that makes their weights."""
import pytest
import torch

from paper_2308_14711_b200 import binding
from paper_2308_14711_b200.binding import FFFLayer, FFFStack

pytestmark = pytest.mark.gpu

DEPTH, LW, B = 4, 12, 300
LONG = 100_000_000                                         # cycles: some hundredths of a second


def weights(D, dtype):
    g = torch.Generator().manual_seed(5)
    n = 1 << DEPTH
    shapes = dict(node_w=(n - 1, D), node_b=(n - 1,), w1=(n, LW, D), b1=(n, LW), w2=(n, D, LW), b2=(n, D))
    return {k: (torch.randn(*s, generator=g) * 0.2).to(dtype).cuda() for k, s in shapes.items()}


def late(tensors):
    """Copies that the current stream makes a while from now; zeros until then."""
    out = {k: torch.zeros_like(t) for k, t in tensors.items()}
    torch.cuda.current_stream().synchronize()
    torch.cuda._sleep(LONG)
    for k, t in tensors.items():
        out[k].copy_(t)
    return out


def plain(w, D, kind):
    return FFFLayer(D, D, DEPTH, LW, "gelu", kind, **w)


def four_bit(w, D, kind):
    c1, s1 = binding.quantize_mx4(w["w1"])
    c2, s2 = binding.quantize_mx4(w["w2"].transpose(1, 2).contiguous())
    return FFFLayer.from_mx4(D, D, DEPTH, LW, "gelu", w["node_w"], w["node_b"], c1, s1, w["b1"], c2, s2, w["b2"])


@pytest.mark.parametrize("make,D,kind", [(plain, 64, "f32"), (plain, 128, "bf16"), (four_bit, 128, "bf16"), (four_bit, 77, "bf16")],
                         ids=["f32", "bf16", "mx4", "mx4_odd"])
def test_layers_take_weights_that_are_on_their_way(make, D, kind):
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    w = weights(D, dtype)
    x = torch.randn(B, D, generator=torch.Generator().manual_seed(6)).to(dtype).cuda()
    torch.cuda.synchronize()
    known = make(w, D, kind)
    y, leaf = known.forward_infer(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        layer = make(late(w), D, kind)
        y2, leaf2 = layer.forward_infer(x)
    torch.cuda.synchronize()
    assert torch.equal(leaf, leaf2) and torch.equal(y, y2)
    known.close()
    layer.close()


def test_stacks_take_vectors_that_are_on_their_way():
    D = 64
    w = weights(D, torch.bfloat16)
    layers = [plain(w, D, "bf16"), plain(w, D, "bf16")]
    g = torch.Generator().manual_seed(7)
    vectors = {k: torch.randn(D, generator=g).bfloat16().cuda() for k in "abcd"}
    x = torch.randn(B, D, generator=g).bfloat16().cuda()
    known = FFFStack(layers, gammas=[vectors["a"], vectors["b"]], betas=[vectors["c"], vectors["d"]])
    y, _ = known.forward(x)
    y = y.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        v = late(vectors)
        stack = FFFStack(layers, gammas=[v["a"], v["b"]], betas=[v["c"], v["d"]])
        y2, _ = stack.forward(x)
    torch.cuda.synchronize()
    assert torch.equal(y, y2)
    known.close()
    stack.close()
