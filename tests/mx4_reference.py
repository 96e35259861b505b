"""Microscaled 4-bit floats in numpy, from the format's definition: what the tests of the library's conversion and layers compare with."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(w):
    """(codes one per byte, scales) of the rows (last axis) of a float array, by distance to every code's value."""
    w = np.asarray(w, dtype=np.float64)
    cols = w.shape[-1]
    nb = (cols + 31) // 32
    codes = np.zeros(w.shape, np.uint8)
    scales = np.zeros(w.shape[:-1] + (nb,), np.uint8)
    for b in range(nb):
        block = w[..., 32 * b:32 * b + 32]
        amax = np.abs(block).max(-1)
        bad = ~np.isfinite(amax)
        e = np.where((amax > 0) & ~bad, np.frexp(np.where(bad, 1.0, amax))[1] - 1 - 2, -127)
        e = np.maximum(e, -127)
        q = np.abs(np.where(bad[..., None], 0.0, block)) * np.exp2(-e.astype(np.float64))[..., None]
        d = np.abs(np.minimum(q, 6.0)[..., None] - E2M1)
        best = d.min(-1, keepdims=True)
        # of two codes at the same distance the even one
        order = np.where(d == best, np.arange(8) % 2 * 8 + np.arange(8), 99)
        c = order.argmin(-1).astype(np.uint8)
        codes[..., 32 * b:32 * b + 32] = np.where(bad[..., None], 0, c | (np.signbit(block).astype(np.uint8) << 3))
        scales[..., b] = np.where(bad, 255, e + 127)
    return codes, scales


def values(codes, scales):
    """float64 values of codes (one per byte)."""
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=-1)[..., :codes.shape[-1]]


def pack(codes):
    if codes.shape[-1] % 2:
        codes = np.concatenate([codes, np.zeros(codes.shape[:-1] + (1,), np.uint8)], -1)
    return np.ascontiguousarray(codes[..., 0::2] | (codes[..., 1::2] << 4))


def unpack(packed, cols):
    return np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[:-1] + (-1,))[..., :cols]
