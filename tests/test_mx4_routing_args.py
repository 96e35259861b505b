"""Argument checks of the 4-bit conversion, of layers made of its codes, and of the routing losses that need no GPU; the numpy reference of
the format against hand cases."""
import ctypes as C

import numpy as np
import pytest

from paper_2308_14711_b200 import binding, build
from tests import mx4_reference as mx

FAKE = 0x1000        # never dereferenced: the checks fail first


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_conversion_refuses_bad_arguments(lib):
    q, d = lib.fff_quantize_mx4, lib.fff_dequantize_mx4
    for dtype in (-1, 2):
        assert q(FAKE, dtype, 1, 1, FAKE, FAKE, None, None) == 1 and d(FAKE, FAKE, dtype, 1, 1, FAKE, None) == 1
    for rows, cols in ((-1, 4), (4, -1)):
        assert q(FAKE, 0, rows, cols, FAKE, FAKE, None, None) == 1 and d(FAKE, FAKE, 0, rows, cols, FAKE, None) == 1
    assert q(FAKE, 0, 1 << 30, 1 << 30, FAKE, FAKE, None, None) == 2 and d(FAKE, FAKE, 0, 1 << 30, 1 << 30, FAKE, None) == 2
    for bad in (dict(src=None), dict(codes=None), dict(scales=None), dict(src=FAKE + 4), dict(codes=FAKE + 1), dict(scales=FAKE + 8), dict(values=FAKE + 2)):
        a = dict(src=FAKE, codes=FAKE, scales=FAKE, values=None, **{})
        a.update(bad)
        assert q(a["src"], 1, 3, 5, a["codes"], a["scales"], a["values"], None) == 1, bad
    for bad in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None), (FAKE + 4, FAKE, FAKE), (FAKE, FAKE + 4, FAKE), (FAKE, FAKE, FAKE + 4)):
        assert d(bad[0], bad[1], 0, 3, 5, bad[2], None) == 1
    assert q(None, 0, 0, 5, None, None, None, None) == 0 and q(None, 0, 5, 0, None, None, None, None) == 0
    assert d(None, None, 0, 0, 5, None, None) == 0


def test_creation_refuses_bad_arguments(lib):
    h = C.c_void_p(1234)

    def create(out=None, D=8, O=4, depth=2, l=2, act=0, nw=FAKE, w1=FAKE, s1=FAKE, w2=FAKE, s2=FAKE):
        return lib.fff_create_mx4(C.byref(h) if out is None else out, D, O, depth, l, act, nw, None, w1, s1, None, w2, s2, None)
    assert create(out=C.POINTER(C.c_void_p)()) == 1
    for bad in (dict(D=0), dict(O=-1), dict(l=0), dict(depth=-1), dict(act=4), dict(nw=None), dict(w1=None), dict(w2=None), dict(s1=None),
                dict(s2=None), dict(w1=FAKE + 4), dict(s1=FAKE + 4), dict(s2=FAKE + 8)):
        assert create(**bad) == 1, bad
        assert h.value is None
    for bad in (dict(depth=21), dict(l=1025)):
        assert create(**bad) == 2 and h.value is None


def test_routing_losses_refuse_dead_handles(lib):
    for h in (None, C.c_void_p(0xdead0)):
        assert lib.fff_balance_loss(h, FAKE, FAKE, None, FAKE, None, None, 1, None) == 6
        assert lib.fff_balance_loss_backward(h, FAKE, None, FAKE, FAKE, FAKE, 1, None) == 6
        assert lib.fff_routing_backward(h, FAKE, FAKE, None, None, None, None, FAKE, 1, None) == 6


def test_reference_by_hand():
    w = np.zeros((1, 33))
    w[0, :10] = [6.0, 5.0, 2.5, 3.5, -0.25, 0.75, 1.25, -1.75, 0.1, 7.0]      # largest 7: exponent 2, scale 1
    w[0, 32] = 0.3                                                             # its own block: exponent -2, scale 2^-4, 4.8 -> 4
    codes, scales = mx.quantize(w)
    assert scales.tolist() == [[127, 123]]
    assert codes[0, :10].tolist() == [7, 6, 4, 6, 8, 2, 2, 12, 0, 7] and codes[0, 32] == 6
    v = mx.values(codes, scales)[0]
    assert v[:10].tolist() == [6.0, 4.0, 2.0, 4.0, 0.0, 1.0, 1.0, -2.0, 0.0, 6.0] and v[32] == 0.25
    assert (mx.unpack(mx.pack(codes), 33) == codes).all()


def test_rows_and_layers_too_long_for_32_bits_are_refused(lib):
    long = (1 << 34) + 1
    assert lib.fff_quantize_mx4(FAKE, 1, 1, long, FAKE, FAKE, None, None) == 2
    assert lib.fff_dequantize_mx4(FAKE, FAKE, 1, 1, long, FAKE, None) == 2
    h = C.c_void_p(1234)
    for D, O in ((2 ** 31 - 1, 8), (8, 2 ** 31 - 1), ((1 << 28) + 1, 1)):
        assert lib.fff_create_mx4(C.byref(h), D, O, 0, 1, 0, None, None, FAKE, FAKE, None, FAKE, FAKE, None) == 2 and h.value is None


def test_values_do_not_lie_over_their_source(lib):
    q = lib.fff_quantize_mx4
    for at in (FAKE, FAKE + 16, FAKE - 16):
        assert q(FAKE, 1, 3, 5, 0x100000, 0x200000, at, None) == 1
