"""4-bit layers whose scales are far from 1: over 2, NaN, or so large that weights are infinite in bfloat16; in every kernel that reads them (a
CTA per token for small batches, tiles of a leaf's tokens, a warp per token for thin leaves), and through the stage call.  Outputs are compared
element by element under the bounds of tests/test_gpu_mx4.py, which are relative to sums of magnitudes and so hold for scales of any size."""
import numpy as np
import pytest
import torch

from paper_2308_14711_b200 import workloads as wl
from tests import mx4_reference as mx
from tests import util
from tests.test_gpu_mx4 import C, expected, layer_of, make

pytestmark = pytest.mark.gpu

FEW, MANY = 300, 2600                                      # a CTA per token up to 592, 4 per SM; tiles, or a warp per token, beyond


def run(layer, x):
    """Outputs by the forward and by the stages, and the leaves."""
    y, leaf = layer.forward_infer(x)
    offsets, perm = layer.leaf_bucketing(leaf)
    staged = layer.grouped_leaf_ff(x, leaf, offsets, perm)
    torch.cuda.synchronize()
    assert layer.last_status() == 0
    host = lambda t: t.float().cpu().numpy().astype(np.float64)
    return host(y), host(staged), leaf.cpu().numpy()


def shifted(codes_scales, by):
    c, s = codes_scales[0], (codes_scales[1].astype(np.int64) + by).astype(np.uint8)
    return c, s, mx.values(c, s)


@pytest.mark.parametrize("B", [FEW, MANY])
@pytest.mark.parametrize("depth,l", [(3, 3), (10, 3), (3, 12), (2, 32), (2, 70), (3, 33)])
@pytest.mark.parametrize("shift1,shift2", [(4, 0), (12, 0), (0, 12), (40, -50), (-60, 70), (30, 60)])
def test_scales_on_both_sides_of_2(shift1, shift2, depth, l, B):
    cfg = C("big", 128, 96, depth, l, "gelu" if shift1 < 20 else "relu", "bf16", B, "normal")
    w, one, two, net, x_host = make(cfg, seed=6)
    one, two = shifted(one, shift1), shifted(two, shift2)
    assert (max(one[1].max(), two[1].max()) > 128) == (max(shift1, shift2) > 6)
    layer = layer_of(cfg, w, one, two)
    y, staged, leaf = run(layer, util.to_device(x_host, "bf16"))
    y_ref, bound = expected(cfg, w, one[2], two[2], x_host, leaf)
    assert np.abs(y_ref).max() < 2.0 ** 120
    for got in (y, staged):
        assert (np.abs(got - y_ref) <= bound).all()
    layer.close()


@pytest.mark.parametrize("B", [FEW, MANY])
@pytest.mark.parametrize("activation", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("l", [3, 12, 32, 70])
def test_a_nan_block_of_w1_makes_its_leaf_nan(l, activation, B):
    """(ReLU, as max(0, .), takes it for 0.)"""
    cfg = C("nan", 128, 64, 2, l, activation, "bf16", B, "normal")
    w, one, two, net, x_host = make(cfg, seed=7)
    bad, other = 2, one[1].copy()
    other[bad, 1, 3] = 255
    layer = layer_of(cfg, w, (one[0], other), two)
    y, staged, leaf = run(layer, util.to_device(x_host, "bf16"))
    ok = leaf != bad
    assert ok.any() and not ok.all()
    y_ref, bound = expected(cfg, w, one[2], two[2], x_host, leaf)
    for got in (y, staged):
        assert np.isnan(got[~ok]).all() and (np.abs(got[ok] - y_ref[ok]) <= bound[ok]).all()
    layer.close()


@pytest.mark.parametrize("B", [FEW, MANY])
@pytest.mark.parametrize("activation", ["gelu", "relu"])
@pytest.mark.parametrize("l", [3, 8, 12, 32, 70])
def test_infinite_output_weights(l, activation, B):
    """Scale 254 makes codes of 2 and more infinite: h times infinity of h's sign, NaN where h is 0, whatever the leaf's width; blocks beside it
    keep their values."""
    cfg = C("inf", 128, 96, 2, l, activation, "bf16", B, "normal")
    w, one, two, net, x_host = make(cfg, seed=8)
    bad, unit = 1, l // 2
    codes, scales = two[0].copy(), two[1].copy()
    scales[bad, unit, 1] = 254                             # outputs 32 to 63
    codes[bad, unit, 32:64] = np.arange(32) % 8 // 4 * 4 + np.arange(32) % 4 * (np.arange(32) % 8 // 4) | np.arange(32) // 16 * 8      # 0 or 2, 3, 4, 6, both signs
    assert set(codes[bad, unit, 32:64] & 7) == {0, 4, 5, 6, 7}
    v2 = mx.values(codes, scales)
    v2 = np.where(np.abs(v2) >= 2.0 ** 128, np.copysign(np.inf, v2), v2)
    layer = layer_of(cfg, w, one, (codes, scales))
    y, staged, leaf = run(layer, util.to_device(x_host, "bf16"))
    assert (leaf == bad).any()
    with np.errstate(invalid="ignore"):
        y_ref, bound = expected(cfg, w, one[2], v2, x_host, leaf)
    finite = np.isfinite(y_ref)
    assert np.isinf(y_ref).any() and (np.isnan(y_ref).any() == (activation == "relu"))
    for got in (y, staged):
        assert (np.abs(got[finite] - y_ref[finite]) <= bound[finite]).all()
        np.testing.assert_array_equal(got[~finite], y_ref[~finite])          # (NaN where NaN, infinities of the same sign)
    layer.close()
