"""Results of calls that are made on another stream (stream=): their memory is nobody else's until both streams are done with it."""
import pytest
import torch

from paper_2308_14711_b200 import binding
from paper_2308_14711_b200.binding import FFFLayer, FFFStack

pytestmark = pytest.mark.gpu

D, DEPTH, LW, B = 64, 6, 8, 700
LONG = 400_000_000                                         # cycles: two tenths of a second and more


@pytest.fixture(params=["module", "ctypes"])
def call(request, monkeypatch):
    """The calls through the CPython module, and as they are made where that has not been built."""
    if request.param == "ctypes":
        monkeypatch.setattr(binding, "torch_call", lambda: None)
    else:
        assert binding.torch_call() is not None


def make():
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: (torch.randn(*s, generator=g) * 0.2).bfloat16().cuda()
    n = 1 << DEPTH
    return FFFLayer(D, D, DEPTH, LW, "gelu", "bf16", rnd(n - 1, D), rnd(n - 1), rnd(n, LW, D), rnd(n, LW), rnd(n, D, LW), rnd(n, D))


def calls():
    """name -> function of a stream that returns what the call allocates."""
    layer = make()
    stack = FFFStack([make(), make()], layer_norm=False, residual=False)
    x = torch.randn(B, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    y, leaf = layer.forward_infer(x)
    _, mix, _ = layer.forward_train(x)
    _, counts, _ = layer.balance_loss(mix, leaf)
    offsets, perm = layer.leaf_bucketing(leaf)
    stack.forward(x)
    layer.last_bucketing(B)
    one, codes = torch.ones(1, device="cuda"), binding.quantize_mx4(x)
    return {
        "forward_infer": lambda s: layer.forward_infer(x, stream=s),
        "forward_train": lambda s: layer.forward_train(x, stream=s),
        "tree_descent": lambda s: (layer.tree_descent(x, stream=s),),
        "leaf_bucketing": lambda s: layer.leaf_bucketing(leaf, stream=s),
        "grouped_leaf_ff": lambda s: (layer.grouped_leaf_ff(x, leaf, offsets, perm, stream=s),),
        "last_bucketing": lambda s: layer.last_bucketing(B, stream=s),
        "stack": lambda s: stack.forward(x, stream=s),
        "balance_loss": lambda s: layer.balance_loss(mix, leaf, stream=s),
        "balance_loss_backward": lambda s: (layer.balance_loss_backward(leaf, counts, one, stream=s),),
        "routing_backward": lambda s: (layer.routing_backward(mix, leaf_idx=leaf, counts=counts, dloss=one, stream=s),),
        "quantize_mx4": lambda s: binding.quantize_mx4(x, want_values=True, stream=s),
        "dequantize_mx4": lambda s: (binding.dequantize_mx4(*codes, D, stream=s),),
    }


NAMES = ["forward_infer", "forward_train", "tree_descent", "leaf_bucketing", "grouped_leaf_ff", "last_bucketing", "stack", "balance_loss",
         "balance_loss_backward", "routing_backward", "quantize_mx4", "dequantize_mx4"]


def places(tensors):
    return [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors if t is not None]


def apart(a, b):
    return all(p1 <= q0 or q1 <= p0 for p0, p1 in a for q0, q1 in b)


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_results(call, name):
    """By their addresses alone.  (A host so slow that the waiting stream is done by the time of a comparison shows nothing there.)"""
    run = calls()[name]
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    torch.cuda.synchronize()
    expected = [t.clone() for t in run(None) if t is not None]
    shapes = [(t.shape, t.dtype) for t in expected]
    again = lambda: [torch.empty(s, dtype=d, device="cuda") for s, d in shapes for _ in range(8)]
    _ = [t + 0 for t in run(side) if t is not None], again()          # (a first time allocates, and loads kernels)
    torch.cuda._sleep(1)
    del _
    torch.cuda.synchronize()
    # what was freed on the current stream may still be in use there: the results lie elsewhere
    old = again()
    torch.cuda._sleep(LONG)
    freed = places(old)
    del old
    got = [t for t in run(side) if t is not None]
    assert apart(places(got), freed) or main.query()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, expected))
    del got
    # dropped while the side stream has still to write them: the current stream's next tensors lie elsewhere
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    got = [t for t in run(side) if t is not None]
    there = places(got)
    del got
    new = again()
    assert apart(places(new), there) or side.query()
    torch.cuda.synchronize()
    del new
    # dropped while the current stream has still to read them: the next call's results lie elsewhere
    got = [t for t in run(side) if t is not None]
    main.wait_stream(side)
    torch.cuda._sleep(LONG)
    read = [t + 0 for t in got]
    there = places(got)
    del got
    got = [t for t in run(side) if t is not None]
    assert apart(places(got), there) or main.query()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(read, expected, got))


def test_other_kinds_of_streams(call):
    """The default stream, whose address is 0, a stream by its address, and something that only has an address."""
    layer = make()
    x = torch.randn(B, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    y, leaf = layer.forward_infer(x)
    side = torch.cuda.Stream()

    class Address:
        cuda_stream = side.cuda_stream

    class Zero:
        cuda_stream = 0
    torch.cuda.synchronize()
    for s in (torch.cuda.default_stream(), torch.cuda.ExternalStream(side.cuda_stream), Address(), Zero()):
        y2, leaf2 = layer.forward_infer(x, stream=s)
        codes = binding.quantize_mx4(x, want_values=True, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(leaf, leaf2)
        assert all(torch.equal(a, b) for a, b in zip(codes, binding.quantize_mx4(x, want_values=True)))
    layer.close()


def test_a_captured_call_on_a_stream_of_the_capture(call):
    """A fork and a join within a capture: results of the forked call are memory of the graph, and every replay writes them."""
    layer = make()
    x = torch.randn(B, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    want = [t.clone() for t in layer.forward_infer(x)] + [t.clone() for t in binding.quantize_mx4(x, want_values=True)]
    other = torch.randn(B, D, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    want_other = [t.clone() for t in layer.forward_infer(other)] + [t.clone() for t in binding.quantize_mx4(other, want_values=True)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        y, leaf = layer.forward_infer(x, stream=side)
        layer.forward_infer(x, stream=side)                # (dropped at once)
        q = binding.quantize_mx4(x, want_values=True, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, leaf) + tuple(q), want))
    keep = x.clone()
    x.copy_(other)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, leaf) + tuple(q), want_other))
    x.copy_(keep)
    del graph
    layer.close()
