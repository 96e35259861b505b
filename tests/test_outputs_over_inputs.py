"""Calls whose outputs would lie over their inputs are refused (addresses alone: nothing is launched)."""
import pytest
import torch

from paper_2308_14711_b200 import binding, build

A = 0x100000                                               # never dereferenced: the checks fail first


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2)])
def test_conversion(lib, dtype, size):
    rows, cols = 48, 64
    n = rows * cols * size
    codes, scales = rows * cols // 2, rows * 2
    free = A + 16 * n
    for at in (A, A + 16, A + n - 16):
        for kw in (dict(codes=at), dict(scales=at), dict(values=at)):
            a = dict(codes=free, scales=2 * free, values=None)
            a.update(kw)
            assert lib.fff_quantize_mx4(A, dtype, rows, cols, a["codes"], a["scales"], a["values"], None) == 1, kw
    for kw in (dict(codes=A - codes + 16), dict(scales=A - scales + 16)):
        a = dict(codes=free, scales=2 * free)
        a.update(kw)
        assert lib.fff_quantize_mx4(A, dtype, rows, cols, a["codes"], a["scales"], None, None) == 1, kw
        assert lib.fff_dequantize_mx4(a["codes"], a["scales"], dtype, rows, cols, A, None) == 1, kw
    for at in (A, A + n - 16):
        assert lib.fff_dequantize_mx4(at, free, dtype, rows, cols, A, None) == 1
        assert lib.fff_dequantize_mx4(free, at, dtype, rows, cols, A, None) == 1


@pytest.mark.gpu
def test_routing_backward(lib):
    depth, B = 3, 40
    z = lambda *s: torch.zeros(s, device="cuda")
    layer = binding.FFFLayer(1, 1, depth, 1, "relu", "f32", z(7, 1), None, z(8, 1, 1), None, z(8, 1, 1), None)
    buf = torch.rand(4 * B * 8, device="cuda")
    mix, up = buf.data_ptr(), buf.data_ptr() + 4 * B * 8
    free = up + 4 * B * 8
    call = lambda dz: lib.fff_routing_backward(layer.handle, mix, up, None, None, None, None, dz, B, None)
    for dz in (mix, mix + 16, up, up + 4 * B * 8 - 16, mix - 4 * B * 7 + 16):
        assert call(dz) == 1
    assert call(free) == 0
    torch.cuda.synchronize()
    # next to the inputs on both sides is next to them
    assert lib.fff_routing_backward(layer.handle, up, up, None, None, None, None, up - 4 * B * 7, B, None) == 0
    torch.cuda.synchronize()
    layer.close()
