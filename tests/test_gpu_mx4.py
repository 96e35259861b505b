"""Microscaled 4-bit floats on the GPU: conversion bit by bit against the definition, layers with such leaf weights against float64.

Tolerance of a layer's outputs, element by element, from the roundings that it makes (u = 2^-24, float32; 2^-8 relative, bf16):
  first product   D + 1 additions in float32 of exact products: |dz| <= (D + 2) u (sum |w1 x| + |b1|);
  activation      slope at most 1.13 (GELU; 1.10 SiLU), evaluated to 16 u relative to max(|z|, 1):
                  |dh| <= 1.13 |dz| + 16 u max(|z|, 1);
  hidden value    kept as a sum of two bf16 values, each within 2^-8 of what it rounds: 2^-16 |h|;
  second product  l + 1 additions: (2 l + 2) u (sum |w2 h| + |b2|) (two summands per hidden value);
  output          2^-8 |y|.
"""
import numpy as np
import pytest
import torch

from oracle import fff_oracle as orc
from paper_2308_14711_b200 import binding, workloads as wl
from paper_2308_14711_b200.binding import FFFError, FFFLayer, FFFStack
from tests import mx4_reference as mx
from tests import util

pytestmark = pytest.mark.gpu

C = wl.FFFConfig
U = 2.0 ** -24


def act(name, v):
    t = torch.from_numpy(np.asarray(v))
    if name == "relu":
        return t.clamp(min=0).numpy()
    if name == "gelu":
        return torch.nn.functional.gelu(t).numpy()
    if name == "gelu_tanh":
        return torch.nn.functional.gelu(t, approximate="tanh").numpy()
    return torch.nn.functional.silu(t).numpy()


def expected(cfg, w, v1, v2, x, leaf):
    """y and the bound of its error, in float64.  v1 [2^d, l, D], v2 [2^d, l, O]: the values of the codes."""
    y, bound = np.empty((x.shape[0], cfg.O)), np.empty((x.shape[0], cfg.O))
    x = x.astype(np.float64)
    for j in np.unique(leaf):
        t = np.flatnonzero(leaf == j)
        b1, b2 = w["b1"][j].astype(np.float64), w["b2"][j].astype(np.float64)
        z = x[t] @ v1[j].T + b1
        h = act(cfg.activation, z)
        y[t] = h @ v2[j] + b2
        dz = (cfg.D + 2) * U * (np.abs(x[t]) @ np.abs(v1[j]).T + np.abs(b1))
        dh = 1.13 * dz + 16 * U * np.maximum(np.abs(z), 1.0) + 2.0 ** -16 * np.abs(h)
        bound[t] = dh @ np.abs(v2[j]) + (2 * cfg.leaf_width + 2) * U * (np.abs(h) @ np.abs(v2[j]) + np.abs(b2))
    return y, bound + 2.0 ** -8 * (np.abs(y) + bound)


def make(cfg, seed, scale_shift=0):
    w = wl.make_weights(cfg, seed)
    c1, s1 = mx.quantize(w["w1"])
    c2, s2 = mx.quantize(np.swapaxes(w["w2"], 1, 2))
    s1 = (s1.astype(np.int64) + scale_shift).astype(np.uint8)
    v1, v2 = mx.values(c1, s1), mx.values(c2, s2)
    net = orc.Net(cfg.D, cfg.O, cfg.depth, cfg.leaf_width, cfg.activation, w["node_w"], w["node_b"], v1.astype(np.float32), w["b1"],
                  np.ascontiguousarray(np.swapaxes(v2, 1, 2)).astype(np.float32), w["b2"])
    src = wl.TokenSource(cfg, seed)
    if cfg.depth:
        wl.enforce_margin(src, lambda rows: orc.path_margin(net, rows, threads=util.ORACLE_THREADS))
    return w, (c1, s1, v1), (c2, s2, v2), net, src.x


def layer_of(cfg, w, one, two):
    dev = {k: util.to_device(w[k], "bf16") for k in ("node_w", "node_b", "b1", "b2")}
    if cfg.depth == 0:
        dev["node_w"] = dev["node_b"] = None
    gpu = lambda a: torch.from_numpy(a).cuda()
    return FFFLayer.from_mx4(cfg.D, cfg.O, cfg.depth, cfg.leaf_width, cfg.activation, dev["node_w"], dev["node_b"], gpu(mx.pack(one[0])),
                             gpu(one[1]), dev["b1"], gpu(mx.pack(two[0])), gpu(two[1]), dev["b2"])


def check(y, leaf, net, cfg, w, one, two, x_host):
    _, leaf_ref = orc.forward_i(net, x_host, threads=util.ORACLE_THREADS)
    np.testing.assert_array_equal(leaf.cpu().numpy(), leaf_ref)
    y_ref, bound = expected(cfg, w, one[2], two[2], x_host, leaf_ref)
    err = np.abs(y.float().cpu().numpy().astype(np.float64) - y_ref)
    assert (err <= bound).all(), f"worst error is {float((err / bound).max()):.2f} times its bound"
    return leaf_ref


# ---- conversion

SPECIAL = [0.0, -0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.5, 6.0, 7.0, 7.99, -0.25, -0.75, -1.25, -2.5, -5.0, -7.5, 1e-3, -1e-3]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (5, 33), (7, 64), (2, 100), (129, 7), (64, 784), (1000, 96), (3, 4099), (70, 40), (90, 200),
                                       (0, 5), (4, 0)])
def test_conversion_is_the_definition(rows, cols, dtype):
    g = np.random.default_rng(rows * 10007 + cols)
    w = g.standard_normal((rows, cols)).astype(np.float32) * np.exp2(g.integers(-140, 120, size=(rows, 1)).astype(np.float32))
    flat = w.reshape(-1)
    for i in range(0, flat.size, 5):
        flat[i] = SPECIAL[(i // 5) % len(SPECIAL)]
    if w.size > 200:
        w[0], w[-1] = 0.0, -0.0                           # a row of zeros of both signs
    if rows >= 64:
        w[1, 3], w[2, cols // 2], w[3, cols - 1] = np.inf, np.nan, -np.inf
        w[5], w[6] = 3.0e38, 1.0e-45
    t = torch.from_numpy(w).to(dtype)
    w = t.float().numpy()
    codes, scales, values = binding.quantize_mx4(t.cuda(), want_values=True)
    c_ref, s_ref = mx.quantize(w)
    assert codes.shape == (rows, (cols + 1) // 2) and scales.shape == (rows, (cols + 31) // 32)
    np.testing.assert_array_equal(scales.cpu().numpy(), s_ref)
    got = mx.unpack(codes.cpu().numpy(), cols) if w.size else np.zeros_like(c_ref)
    np.testing.assert_array_equal(got, c_ref)
    if cols % 2 and w.size:
        assert (codes.cpu().numpy()[:, -1] >> 4 == 0).all()
    # the values are exact in either type wherever they are not subnormal; there they are the nearest ones
    v_ref = torch.from_numpy(mx.values(c_ref, s_ref)).to(dtype)
    assert torch.equal(torch.nan_to_num(values.cpu(), nan=7e30), torch.nan_to_num(v_ref, nan=7e30))
    again = binding.dequantize_mx4(codes, scales, cols, dtype)
    assert torch.equal(torch.nan_to_num(again, nan=7e30), torch.nan_to_num(values, nan=7e30))
    c2, s2 = binding.quantize_mx4(t.cuda())
    assert torch.equal(c2, codes) and torch.equal(s2, scales)


def test_every_code_and_scale_is_read_back():
    codes = np.tile(np.arange(16, dtype=np.uint8), 2)[None].repeat(256, 0)
    scales = np.arange(256, dtype=np.uint8)[:, None]
    for dtype in (torch.float32, torch.bfloat16):
        got = binding.dequantize_mx4(torch.from_numpy(mx.pack(codes)).cuda(), torch.from_numpy(scales).cuda(), 32, dtype).cpu()
        ref = torch.from_numpy(mx.values(codes, scales)).to(dtype)
        assert torch.equal(torch.nan_to_num(got, nan=7e30, posinf=8e30, neginf=-8e30), torch.nan_to_num(ref, nan=7e30, posinf=8e30, neginf=-8e30))


def test_conversion_writes_nothing_past_its_arrays():
    rows, cols = 37, 45
    w = torch.randn(rows, cols, device="cuda")
    cb, nb = (cols + 1) // 2, (cols + 31) // 32
    codes = torch.full((rows * cb + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows * nb + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    values = torch.full((rows * cols + 64,), -7.0, device="cuda")
    L = binding.lib()
    assert L.fff_quantize_mx4(w.data_ptr(), 0, rows, cols, codes.data_ptr(), scales.data_ptr(), values.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert (codes[rows * cb:] == 0xA5).all() and (scales[rows * nb:] == 0xA5).all() and (values[rows * cols:] == -7.0).all()
    c, s, v = binding.quantize_mx4(w, want_values=True)
    assert torch.equal(codes[:rows * cb], c.flatten()) and torch.equal(scales[:rows * nb], s.flatten()) and torch.equal(values[:rows * cols], v.flatten())


# ---- layers

CASES = [
    C("l8", 256, 128, 6, 8, "gelu", "bf16", 3001, "normal"),               # narrowest leaf of the tensor-core kernel
    C("l12", 768, 768, 4, 12, "gelu", "bf16", 1500, "layernorm"),          # tiles of 64 rows
    C("l16", 128, 256, 7, 16, "silu", "bf16", 4099, "clusters"),           # a few large buckets, many empty leaves
    C("l32", 512, 320, 5, 32, "gelu_tanh", "bf16", 777, "normal"),
    C("l33", 192, 64, 3, 33, "relu", "bf16", 300, "normal"),               # two K-blocks, the second almost empty
    C("l64", 128, 272, 3, 64, "relu", "bf16", 2000, "normal"),
    C("l96", 64, 72, 2, 96, "gelu", "bf16", 129, "normal"),
    C("l200", 96, 40, 1, 200, "gelu", "bf16", 200, "normal"),              # hidden values of a tile in 64 KB
    C("l1024", 48, 24, 0, 1024, "gelu", "bf16", 70, "normal"),             # widest, a plain feedforward layer
    C("odd", 77, 51, 4, 11, "gelu", "bf16", 257, "normal"),                # no row on a 16-byte boundary
    C("mult8", 104, 88, 5, 24, "gelu", "bf16", 900, "normal"),             # rows of 16-byte vectors, not of 32
    C("tiny", 1, 1, 3, 9, "gelu", "bf16", 33, "normal", node_bias_std=0.5),
    C("one_leaf", 256, 256, 0, 32, "silu", "bf16", 4000, "normal"),
    C("one_token", 1024, 1024, 5, 32, "gelu", "bf16", 1, "normal"),
    C("two_stages", 256, 256, 10, 16, "gelu", "bf16", 20000, "normal"),    # lists between the descent stages
    C("many_leaves", 128, 64, 12, 8, "gelu", "bf16", 3000, "normal"),      # more leaves than lists are read for
    C("thin1", 768, 768, 10, 1, "gelu", "bf16", 1500, "normal"),           # CUDA cores; the walk's last levels in the leaf kernel
    C("thin3", 200, 136, 6, 3, "relu", "bf16", 1000, "normal"),            # ... behind a bucketing
    C("thin7_odd", 45, 33, 3, 7, "gelu", "bf16", 100, "normal"),
    C("thin2_wide", 1500, 1501, 2, 2, "silu", "bf16", 40, "normal"),
]


@pytest.mark.parametrize("cfg", CASES, ids=lambda c: c.name)
def test_forward_matches_float64(cfg):
    w, one, two, net, x_host = make(cfg, seed=4)
    layer = layer_of(cfg, w, one, two)
    x = util.to_device(x_host, "bf16")
    first = None
    for _ in range(2):
        y, leaf = layer.forward_infer(x)
        torch.cuda.synchronize()
        assert layer.last_status() == 0 and layer.last_launch_count() > 0
        leaf_ref = check(y, leaf, net, cfg, w, one, two, x_host)
        assert first is None or torch.equal(y, first)
        first = y.clone()
    off_ref, perm_ref = orc.bucket(leaf_ref, cfg.n_leaves)
    off, perm = layer.last_bucketing(cfg.B)
    np.testing.assert_array_equal(off.cpu().numpy(), off_ref)
    np.testing.assert_array_equal(perm.cpu().numpy(), perm_ref)
    # the stages on the same handle
    leaf2 = layer.tree_descent(x)
    off, perm = layer.leaf_bucketing(leaf2)
    y2 = layer.grouped_leaf_ff(x, leaf2, off, perm)
    check(y2, leaf2, net, cfg, w, one, two, x_host)
    # host buffers, and a smaller batch on the grown workspace
    xh, yh = x.cpu().pin_memory(), torch.empty((cfg.B, cfg.O), dtype=torch.bfloat16).pin_memory()
    lh = torch.empty(cfg.B, dtype=torch.int32).pin_memory()
    layer.forward_infer_host(xh, yh, lh)
    check(yh, lh, net, cfg, w, one, two, x_host)
    n = (cfg.B + 2) // 3
    y3, leaf3 = layer.forward_infer(x[:n].contiguous())
    check(y3, leaf3, net, cfg, w, one, two, x_host[:n])
    layer.close()


@pytest.mark.parametrize("cfg", [C("big32", 128, 96, 3, 32, "relu", "bf16", 300, "normal"), C("big12", 64, 64, 2, 12, "relu", "bf16", 90, "normal"),
                                 C("big3", 128, 96, 3, 3, "relu", "bf16", 300, "normal")], ids=lambda c: c.name)
@pytest.mark.parametrize("shift", [-60, 4, 8, 40])
def test_scales_of_all_sizes(cfg, shift):
    """Scales over 2 take a second product; ones far from it neither overflow nor vanish on the way."""
    w, one, two, net, x_host = make(cfg, seed=6, scale_shift=shift)
    assert (one[1].max() > 128) == (shift > 6)
    layer = layer_of(cfg, w, one, two)
    y, leaf = layer.forward_infer(util.to_device(x_host, "bf16"))
    check(y, leaf, net, cfg, w, one, two, x_host)
    layer.close()


@pytest.mark.parametrize("l", [3, 12, 32])
def test_a_nan_block_reaches_its_leaf_alone(l):
    cfg = C("nan", 128, 64, 2, l, "relu", "bf16", 400, "normal")
    w, one, two, net, x_host = make(cfg, seed=7)
    bad, other = 2, one[1].copy()
    other[bad, 1, 3] = 255
    layer = layer_of(cfg, w, (one[0], other, one[2]), two)
    y, leaf = layer.forward_infer(util.to_device(x_host, "bf16"))
    y, leaf = y.float().cpu().numpy(), leaf.cpu().numpy()
    assert (leaf == bad).any() and (leaf != bad).any()
    # (ReLU of a NaN is 0 in this library, as fmax makes it: the outputs of that leaf are finite or NaN, never another leaf's)
    y_ref, bound = expected(cfg, w, one[2], two[2], x_host, leaf)
    ok = leaf != bad
    assert (np.abs(y[ok] - y_ref[ok]) <= bound[ok]).all()
    layer.close()
    # in the output weights: block 1 of unit 1 covers outputs 32 to 63
    other = two[1].copy()
    other[bad, 1, 1] = 255
    layer = layer_of(cfg, w, one, (two[0], other, two[2]))
    y, _ = layer.forward_infer(util.to_device(x_host, "bf16"))
    y = y.float().cpu().numpy()
    assert np.isnan(y[~ok][:, 32:]).all() and np.isfinite(y[~ok][:, :32]).all()
    assert (np.abs(y[ok] - y_ref[ok]) <= bound[ok]).all()
    layer.close()


def test_a_nan_token_and_an_infinite_one_stay_in_their_rows():
    cfg = C("rows", 128, 64, 2, 16, "gelu", "bf16", 200, "normal")
    w, one, two, net, x_host = make(cfg, seed=8)
    layer = layer_of(cfg, w, one, two)
    x = util.to_device(x_host, "bf16")
    clean, leaf = layer.forward_infer(x)
    clean, leaf = clean.clone(), leaf.clone()
    x[17] = float("nan")
    x[55, 3] = float("inf")
    y, got = layer.forward_infer(x)
    keep = torch.ones(cfg.B, dtype=torch.bool, device="cuda")
    keep[17] = keep[55] = False
    assert torch.equal(y[keep], clean[keep]) and torch.equal(got[keep], leaf[keep])
    assert torch.isnan(y[17]).all() and ((got >= 0) & (got < cfg.n_leaves)).all()
    layer.close()


def test_forward_on_another_stream_captured_and_replayed():
    cfg = C("graph", 256, 128, 5, 12, "gelu", "bf16", 700, "normal")
    w, one, two, net, x_host = make(cfg, seed=9)
    layer = layer_of(cfg, w, one, two)
    layer.reserve(cfg.B)
    x = util.to_device(x_host, "bf16")
    y, leaf = torch.empty((cfg.B, cfg.O), dtype=torch.bfloat16, device="cuda"), torch.empty(cfg.B, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    layer.forward_infer(x, y, leaf, stream=side)
    side.synchronize()
    check(y, leaf, net, cfg, w, one, two, x_host)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.forward_infer(x, y, leaf)
    order = torch.randperm(cfg.B, generator=torch.Generator().manual_seed(1))
    y.zero_()
    x.copy_(util.to_device(x_host[order.numpy()], "bf16"))
    graph.replay()
    torch.cuda.synchronize()
    check(y, leaf, net, cfg, w, one, two, x_host[order.numpy()])
    del graph
    layer.close()


def test_a_stack_of_4_bit_layers():
    cfg = C("stack", 256, 256, 4, 16, "gelu", "bf16", 500, "layernorm")
    parts = [make(cfg, seed=20 + k) for k in range(2)]
    layers = [layer_of(cfg, p[0], p[1], p[2]) for p in parts]
    stack = FFFStack(layers, layer_norm=False, residual=False)
    x = util.to_device(parts[0][4], "bf16")
    y, leaf = stack.forward(x)
    mid, leaf0 = layers[0].forward_infer(x)
    end, leaf1 = layers[1].forward_infer(mid)
    assert torch.equal(y, end) and torch.equal(leaf[0], leaf0) and torch.equal(leaf[1], leaf1)
    stack.close()
    for l in layers:
        l.close()


# ---- refusals

def test_layers_that_are_refused():
    cfg = C("bad", 64, 64, 1, 8, "relu", "bf16", 4, "normal")
    w, one, two, _, _ = make(cfg, seed=1)
    layer = layer_of(cfg, w, one, two)
    for path in ("warp", "tensor", "fused"):
        with pytest.raises(FFFError) as e:
            layer.set_path(path)
        assert e.value.status == 2
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(FFFError) as e:
        layer.forward_train(x)
    assert e.value.status == 2
    with pytest.raises(ValueError):
        layer.forward_infer(x.float())
    layer.close()
    with pytest.raises(ValueError):                        # W2 as fff_create wants it
        layer_of(cfg.__class__("bad", 64, 62, 1, 8, "relu", "bf16", 4, "normal"), w, one, two)
    wide = C("wide", 8, 8, 0, 1025, "relu", "bf16", 4, "normal")
    w, one, two, _, _ = make(wide, seed=1)
    with pytest.raises(FFFError) as e:
        layer_of(wide, w, one, two)
    assert e.value.status == 2


@pytest.mark.parametrize("way", ["module", "ctypes"])
def test_conversions_that_are_refused(way, monkeypatch):
    if way == "ctypes":
        monkeypatch.setattr(binding, "torch_call", lambda: None)
    with pytest.raises(ValueError):
        binding.quantize_mx4(torch.zeros(4, 4, dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        binding.quantize_mx4(torch.zeros(4, 8, device="cuda")[:, ::2])
    with pytest.raises(ValueError):
        binding.quantize_mx4(torch.zeros(4, 4))
    c, s = binding.quantize_mx4(torch.zeros(4, 40, device="cuda"))
    with pytest.raises(ValueError):
        binding.dequantize_mx4(c, s, 42)
    with pytest.raises(ValueError):
        binding.dequantize_mx4(c, s.int(), 40)


# ---- rows that are no 16-byte vectors, and rows of several chunks

ODD_CASES = [
    C("odd_tiles", 333, 213, 6, 12, "gelu", "bf16", 3001, "normal"),
    C("odd_in", 1021, 64, 4, 24, "relu", "bf16", 3000, "layernorm"),
    C("odd_out", 64, 203, 3, 40, "silu", "bf16", 2500, "normal"),
    C("even_rows", 250, 122, 5, 32, "gelu", "bf16", 2800, "normal"),       # of 4-byte words
    C("odd_thin", 141, 77, 5, 5, "gelu", "bf16", 3000, "normal"),
    C("few_columns", 3, 5, 2, 9, "gelu", "bf16", 5000, "normal", node_bias_std=0.5),
    C("one_column", 1, 1, 1, 8, "relu", "bf16", 4000, "normal", node_bias_std=0.5),
    C("odd_plain", 95, 97, 0, 33, "gelu", "bf16", 2000, "normal"),
    C("odd_two_stages", 129, 65, 10, 16, "gelu", "bf16", 20001, "normal"),  # host buffers in chunks
    C("chunks", 2100, 40, 3, 16, "gelu", "bf16", 1500, "normal"),          # x in three chunks, the last of 52 columns
    C("chunks_wide", 1100, 72, 2, 70, "relu", "bf16", 1400, "normal"),
    C("chunks_odd", 1111, 39, 3, 12, "silu", "bf16", 1500, "normal"),
]


@pytest.mark.parametrize("cfg", ODD_CASES, ids=lambda c: c.name)
def test_rows_of_any_length(cfg):
    test_forward_matches_float64(cfg)


@pytest.mark.parametrize("l", [16, 24, 40])
@pytest.mark.parametrize("D", [1100, 1104])
def test_an_infinity_in_an_earlier_chunk_stays_where_it_is(D, l):
    """Columns behind the last chunk's are nobody's: an infinite value of an earlier chunk does not turn up there (times zero: NaN)."""
    cfg = C("inf", D, 48, 0, l, "relu", "bf16", 1500, "normal")
    w = wl.make_weights(cfg, 3)
    w["w1"][:, :, 100] = 1.0                               # column 100 of the second chunk is behind the end
    w["w2"] = np.abs(w["w2"]) + 0.5
    c1, s1 = mx.quantize(w["w1"])
    c2, s2 = mx.quantize(np.swapaxes(w["w2"], 1, 2))
    v1, v2 = mx.values(c1, s1), mx.values(c2, s2)
    assert (v1[:, :, 100] > 0).all() and (v2 > 0).all()
    layer = layer_of(cfg, w, (c1, s1), (c2, s2))
    x = torch.from_numpy(np.random.default_rng(5).standard_normal((cfg.B, cfg.D)).astype(np.float32)).bfloat16().cuda()
    clean, _ = layer.forward_infer(x)
    clean = clean.clone()
    x[7, 100] = float("inf")
    y, _ = layer.forward_infer(x)
    keep = torch.arange(cfg.B, device="cuda") != 7
    assert (y[7] == float("inf")).all() and torch.equal(y[keep], clean[keep])
    layer.close()


@pytest.mark.parametrize("D,O,l", [(77, 51, 16), (130, 35, 9), (64, 7, 40), (61, 64, 3)])
def test_odd_rows_keep_to_themselves(D, O, l):
    """A NaN token stays in its row, and nothing behind the last row is written."""
    cfg = C("rows", D, O, 2, l, "gelu", "bf16", 2500, "normal")
    w, one, two, net, x_host = make(cfg, seed=8)
    layer = layer_of(cfg, w, one, two)
    x = util.to_device(x_host, "bf16")
    clean, leaf = layer.forward_infer(x)
    check(clean, leaf, net, cfg, w, one, two, x_host)
    clean = clean.clone()
    bad = [0, 17, 1003, cfg.B - 1]
    x[bad] = float("nan")
    flat = torch.full((cfg.B * O + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    y = flat[:cfg.B * O].view(cfg.B, O)
    layer.forward_infer(x, y, torch.empty(cfg.B, dtype=torch.int32, device="cuda"))
    keep = torch.ones(cfg.B, dtype=torch.bool, device="cuda")
    keep[bad] = False
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[bad]).all() and (flat[cfg.B * O:] == 7.0).all()
    layer.close()


def test_odd_rows_captured_and_in_a_stack():
    cfg = C("graph", 77, 77, 5, 12, "gelu", "bf16", 2500, "normal")
    w, one, two, net, x_host = make(cfg, seed=9)
    layer = layer_of(cfg, w, one, two)
    x = util.to_device(x_host, "bf16")
    y, leaf = torch.empty((cfg.B, cfg.O), dtype=torch.bfloat16, device="cuda"), torch.empty(cfg.B, dtype=torch.int32, device="cuda")
    layer.forward_infer(x, y, leaf)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward_infer(x, y, leaf)
    order = np.random.default_rng(1).permutation(cfg.B)
    y.zero_()
    x.copy_(util.to_device(x_host[order], "bf16"))
    graph.replay()
    torch.cuda.synchronize()
    check(y, leaf, net, cfg, w, one, two, x_host[order])
    stack = FFFStack([layer, layer_of(cfg, w, one, two)], layer_norm=False, residual=False)
    end, leaves = stack.forward(x)
    again, last = layer.forward_infer(y.clone())
    assert torch.equal(end, again) and torch.equal(leaves[0], leaf) and torch.equal(leaves[1], last)
    stack.close()
    del graph
    layer.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 2), (1, 7), (1, 9), (2, 3), (3, 5), (8, 1), (9, 1), (300, 1), (517, 3), (33, 34), (40, 36), (65, 37), (31, 66),
                                       (17, 255), (16, 1002), (23, 1001), (200, 44)])
def test_conversion_of_rows_that_start_anywhere(rows, cols, dtype):
    """Every place of a row's start in 16 bytes, ends of the array inside a vector, and nothing written behind it."""
    g = torch.Generator().manual_seed(rows * 131 + cols)
    w = torch.randn(rows, cols, generator=g).to(dtype).cuda()
    codes, scales, values = binding.quantize_mx4(w, want_values=True)
    c_ref, s_ref = mx.quantize(w.float().cpu().numpy())
    np.testing.assert_array_equal(scales.cpu().numpy(), s_ref)
    np.testing.assert_array_equal(mx.unpack(codes.cpu().numpy(), cols), c_ref)
    assert torch.equal(values.cpu(), torch.from_numpy(mx.values(c_ref, s_ref)).to(dtype))
    cb, nb = (cols + 1) // 2, (cols + 31) // 32
    c = torch.full((rows * cb + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((rows * nb + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    v = torch.full((rows * cols + 64,), -7.0, dtype=dtype, device="cuda")
    L, kind = binding.lib(), 0 if dtype == torch.float32 else 1
    assert L.fff_quantize_mx4(w.data_ptr(), kind, rows, cols, c.data_ptr(), s.data_ptr(), v.data_ptr(), None) == 0
    torch.cuda.synchronize()
    for got, want, n, fill in ((c, codes, rows * cb, 0xA5), (s, scales, rows * nb, 0xA5), (v, values, rows * cols, -7.0)):
        assert torch.equal(got[:n], want.flatten()) and (got[n:] == fill).all()
    v.fill_(-7.0)
    assert L.fff_dequantize_mx4(c.data_ptr(), s.data_ptr(), kind, rows, cols, v.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(v[:rows * cols], values.flatten()) and (v[rows * cols:] == -7.0).all()
