"""4-bit layers with every tuning switch off, in recorded stacks, with very long rows, and two of them at once on two streams."""
import numpy as np
import pytest
import torch

from paper_2308_14711_b200 import binding
from paper_2308_14711_b200.binding import FFFStack
from tests import util
from tests.test_gpu_mx4 import C, check, layer_of, make

pytestmark = pytest.mark.gpu

SHAPES = [
    C("few", 128, 96, 5, 12, "gelu", "bf16", 300, "normal"),
    C("tiles", 256, 128, 6, 32, "silu", "bf16", 4000, "normal"),
    C("odd", 173, 99, 6, 24, "gelu", "bf16", 3000, "normal"),
    C("wide", 128, 64, 3, 48, "relu", "bf16", 2500, "normal"),
    C("two_stages", 128, 64, 10, 16, "gelu", "bf16", 9000, "normal"),
    C("thin", 128, 64, 9, 3, "gelu", "bf16", 1500, "normal"),
    C("thin_buckets", 136, 64, 5, 2, "gelu_tanh", "bf16", 2000, "normal"),
]


@pytest.mark.parametrize("cfg", SHAPES, ids=lambda c: c.name)
def test_every_switch(cfg):
    w, one, two, net, x_host = make(cfg, seed=12)
    layer = layer_of(cfg, w, one, two)
    x = util.to_device(x_host, "bf16")
    for key in binding.TUNING:
        layer.set_tuning(key, False)
        for part in (x, x[:97].contiguous()):
            y, leaf = layer.forward_infer(part)
            torch.cuda.synchronize()
            assert layer.last_status() == 0
            check(y, leaf, net, cfg, w, one, two, x_host[:part.shape[0]])
        layer.set_tuning(key, True)
    for key in binding.TUNING:                             # and all at once
        layer.set_tuning(key, False)
    y, leaf = layer.forward_infer(x)
    check(y, leaf, net, cfg, w, one, two, x_host)
    layer.close()


@pytest.mark.parametrize("width", [128, 77])
def test_a_recorded_stack(width):
    cfg = C("stack", width, width, 5, 12, "gelu", "bf16", 2500, "normal")
    parts = [make(cfg, seed=30 + k) for k in range(2)]
    layers = [layer_of(cfg, p[0], p[1], p[2]) for p in parts]
    stack = FFFStack(layers, layer_norm=True, residual=True)
    x = util.to_device(parts[0][4], "bf16")
    y, leaf = torch.empty_like(x), torch.empty((2, cfg.B), dtype=torch.int32, device="cuda")
    stack.forward(x, y, leaf)
    torch.cuda.synchronize()
    want = y.clone(), leaf.clone()
    stack.set_graph(True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    replayed = False
    for _ in range(4):
        y.zero_()
        side.wait_stream(torch.cuda.current_stream())
        stack.forward(x, y, leaf, stream=side)
        side.synchronize()
        replayed |= stack.last_was_replay()
        assert torch.equal(y, want[0]) and torch.equal(leaf, want[1])
    assert replayed
    # a larger batch through one layer replaces its workspace: the recording is not replayed on the old one
    layers[0].forward_infer(util.to_device(np.tile(parts[0][4], (3, 1)), "bf16"))
    torch.cuda.synchronize()
    y.zero_()
    torch.cuda.synchronize()
    stack.forward(x, y, leaf, stream=side)
    side.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(leaf, want[1])
    stack.close()
    for l in layers:
        l.close()


@pytest.mark.parametrize("cfg", [C("long_in", 20011, 40, 2, 16, "gelu", "bf16", 700, "normal"), C("long_in_few", 20016, 40, 2, 40, "gelu", "bf16", 40, "normal"),
                                 C("long_out", 64, 20013, 2, 16, "gelu", "bf16", 700, "normal"), C("long_thin", 60000, 24, 1, 2, "relu", "bf16", 300, "normal"),
                                 C("very_long_few", 60000, 40, 1, 12, "silu", "bf16", 30, "normal")], ids=lambda c: c.name)
def test_long_rows(cfg):
    w, one, two, net, x_host = make(cfg, seed=13)
    layer = layer_of(cfg, w, one, two)
    y, leaf = layer.forward_infer(util.to_device(x_host, "bf16"))
    check(y, leaf, net, cfg, w, one, two, x_host)
    layer.close()


def test_two_layers_on_two_streams_at_once():
    cfgs = [C("a", 256, 128, 6, 32, "gelu", "bf16", 6000, "normal"), C("b", 173, 99, 6, 24, "gelu", "bf16", 5000, "normal")]
    made = [make(c, seed=14) for c in cfgs]
    layers = [layer_of(c, *m[:3]) for c, m in zip(cfgs, made)]
    xs = [util.to_device(m[4], "bf16") for m in made]
    for l, x in zip(layers, xs):
        l.forward_infer(x)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cfgs]
    out = [[], []]
    for _ in range(10):
        for k in (0, 1):
            out[k].append(layers[k].forward_infer(xs[k], stream=streams[k]))
    torch.cuda.synchronize()
    for k in (0, 1):
        check(*out[k][0], made[k][3], cfgs[k], *made[k][:3], made[k][4])
        for y, leaf in out[k][1:]:
            assert torch.equal(y, out[k][0][0]) and torch.equal(leaf, out[k][0][1])
        layers[k].close()
