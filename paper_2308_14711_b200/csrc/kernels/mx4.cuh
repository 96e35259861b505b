// Microscaled 4-bit floating point: conversion, weight images, and the leaf networks on such weights.
//
// A row of numbers is cut into blocks of 32; a block has one power of two for a scale, stored as a biased exponent (e8m0: 2^(s - 127),
// 255 = NaN), and 32 codes of 4 bits (e2m1: sign, two exponent bits, one mantissa bit: 0, 1/2, 1, 3/2, 2, 3, 4, 6).  A code stands for
// its value times the scale of its block.  A block of largest magnitude a gets the scale 2^(floor(log2 a) - 2), which puts a between 4
// and 8; every element is then rounded to the nearest code, ties to the even one, what exceeds 6 to 6 (OCP Microscaling Formats 1.0).
//
// Both leaf matrices are stored with blocks along the long axis, W1 [l, D] and W2 transposed [l, O]: leaves are thin, and blocks along l
// would be mostly scales.  Every such weight is exactly a bf16 value (one mantissa bit, an exponent), so the products are those of a bf16
// layer: expanded in registers on the way into mma.sync, accumulated in float32.
#pragma once

#include <cuda_fp4.h>

#include "common.cuh"
#include "ptx.cuh"
#include "token_block.cuh"

namespace fff {

constexpr int kMxBlock = 32;
__host__ __device__ inline int64_t mx_code_bytes(int64_t cols) { return (cols + 1) / 2; }
__host__ __device__ inline int64_t mx_scales(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }

// ---- conversion ------------------------------------------------------------------------------------

// 2^(s - 127) as float32 (s = 0: the subnormal 2^-127; 255: NaN).
__device__ __forceinline__ float mx_scale(int s) {
    return s == 255 ? __uint_as_float(0x7fffffffu) : s == 0 ? __uint_as_float(0x00400000u) : __uint_as_float((unsigned)s << 23);
}
// The e2m1 value of a code: its exponent and mantissa bits on top of a float32's, which lacks a factor 2^126 (subnormals included).
__device__ __forceinline__ float mx_code_value(unsigned code) {
    return __uint_as_float(((code & 8u) << 28) | ((code & 7u) << 22)) * 8.507059173023462e37f;
}
// Scale of a block of largest magnitude a, by its float32 bits (sign cleared): the exponent less two, 0 at least.  255 where a is not finite.
__device__ __forceinline__ int mx_block_scale(unsigned a) { return a >= 0x7f800000u ? 255 : max((int)(a >> 23) - 2, 0); }

template <typename T> __device__ __forceinline__ float load_float(const T* p) { return Elem<T>::to_float(*p); }

// How rows lie: whole blocks, i.e. one long run of 16-byte vectors; whole groups of eight columns, so that vectors start everywhere but
// blocks may be cut; anything.
enum : int { kMxWhole = 0, kMxGroups = 1, kMxAny = 2 };
constexpr int kMxAtOnce = 2;

// unit / d and its remainder; 32-bit where the numbers are (a 64-bit division is a call of 100 instructions).
__device__ __forceinline__ int64_t mx_divide(int64_t unit, uint32_t d, bool small, uint32_t& rest) {
    if (small) {
        const uint32_t q = (uint32_t)unit / d;
        rest = (uint32_t)unit - q * d;
        return q;
    }
    const int64_t q = unit / d;
    rest = (uint32_t)(unit - q * d);
    return q;
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// Scales in an image: a byte holds the exponent field of 2^126 2^(s - 127), which also makes up for the missing factor: s + 126, one
// product per register.  A layer with a scale over 2 (s > 128; a block with a weight of 8 or more, or the NaN scale) keeps s itself,
// and its kernels multiply twice (kBig).
__device__ __forceinline__ uint32_t mx_mul1(uint32_t byte, bool big) { return (big ? min(byte, 128u) + 126u : byte) * 0x00800080u; }
__device__ __forceinline__ uint32_t mx_mul2(uint32_t byte) {
    return byte == 255 ? 0x7fff7fffu : (byte > 128u ? byte - 1u : 127u) * 0x00800080u;
}
// Two bf16 values, infinities and NaN as zeros.
__device__ __forceinline__ uint32_t mx_finite(uint32_t two) { return two & ~__vcmpeq2(two & 0x7f807f80u, 0x7f807f80u); }
// The values of a word's first n codes, times the scale of byte s.  `each`: elements that a store may have, as n and the place are
// multiples of them: 8 or 4; or 1, and then neighbours go in pairs where they lie on an even place.
template <typename T>
__device__ __forceinline__ void mx_write_values(T* __restrict__ to, uint32_t word, int s, int n, int each) {
    if constexpr (sizeof(T) == 2) {
        // two codes' sign, exponent and mantissa bits to a bf16's, which lacks a factor 2^126; products of powers of two, so that rounded
        // once at most (where the value is subnormal)
        const uint32_t f1 = mx_mul1((uint32_t)s, true), f2 = mx_mul2((uint32_t)s);
        uint32_t o[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t t = word >> (8 * p) & 0xffu, x = t | t << 12;      // nibbles at bits 0 and 16
            o[p] = mul_bf16x2((x & 0x00070007u) << 6 | (x & 0x00080008u) << 12, f1);
        }
        if (s > 128) {
#pragma unroll
            for (int p = 0; p < 4; ++p) o[p] = mul_bf16x2(o[p], f2);
        }
        if (each == 8) {
            __stcs(reinterpret_cast<uint4*>(to), make_uint4(o[0], o[1], o[2], o[3]));
        } else if (each == 4) {
            if (n > 0) *reinterpret_cast<uint2*>(to) = make_uint2(o[0], o[1]);
            if (n > 4) *reinterpret_cast<uint2*>(to + 4) = make_uint2(o[2], o[3]);
        } else {
            const bool odd = reinterpret_cast<uintptr_t>(to) >> 1 & 1;
            uint16_t* one = reinterpret_cast<uint16_t*>(to);
            if (odd && n > 0) one[0] = (uint16_t)o[0];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int e = 2 * p + odd;
                const uint32_t two = odd ? (p < 3 ? __funnelshift_r(o[p], o[p + 1], 16) : o[p] >> 16) : o[p];
                if (e + 1 < n) *reinterpret_cast<uint32_t*>(one + e) = two;
                else if (e < n) one[e] = (uint16_t)two;
            }
        }
    } else {
        const float scale = mx_scale(s);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = mx_code_value(word >> (4 * e)) * scale;
        if (each >= 4) {
            if (n > 0) __stcs(reinterpret_cast<float4*>(to), make_float4(o[0], o[1], o[2], o[3]));
            if (n > 4) __stcs(reinterpret_cast<float4*>(to) + 1, make_float4(o[4], o[5], o[6], o[7]));
        } else {
            const bool odd = reinterpret_cast<uintptr_t>(to) >> 2 & 1;
            if (odd && n > 0) to[0] = o[0];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int e = 2 * p + odd;
                const float a = odd ? o[2 * p + 1] : o[2 * p], b = odd ? (p < 3 ? o[2 * p + 2] : 0.0f) : o[2 * p + 1];
                if (e + 1 < n) *reinterpret_cast<float2*>(to + e) = make_float2(a, b);
                else if (e < n) to[e] = a;
            }
        }
    }
}
__device__ __forceinline__ int mx_store_elements(int64_t cols) { return cols % 4 == 0 ? 4 : 1; }

// Eight bf16 values from value `skip` of two neighbouring 16-byte vectors on.
__device__ __forceinline__ void mx_shift(const uint4 (&raw)[2], int skip, float (&v)[8]) {
    uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
    for (int k = 0; k < 6; ++k) w[k] = skip & 4 ? w[k + 2] : w[k];
#pragma unroll
    for (int k = 0; k < 5; ++k) w[k] = skip & 2 ? w[k + 1] : w[k];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = skip & 1 ? __funnelshift_r(w[k], w[k + 1], 16) : w[k];
    Elem<__nv_bfloat16>::unpack(make_uint4(w[0], w[1], w[2], w[3]), v);
}

// Eight elements per thread, four threads per block.  Bound: HBM, reads and writes in turn, and issue slots (69 % busy): 65 536 rows of 1024
// bf16 values with the values written back 55.0 us (84 % of 6551 GB/s).
template <typename T, int kRows>
__global__ void __launch_bounds__(256)
k_quantize_mx4(const T* __restrict__ src, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, T* __restrict__ values, int64_t rows,
               int64_t cols)
{
    pdl_trigger();
    pdl_wait();
    const int64_t nb = mx_scales(cols), cb = mx_code_bytes(cols), total = rows * nb * 4;
    const int64_t step = (int64_t)gridDim.x * blockDim.x;
    const bool small = total + 4 * step < ((int64_t)1 << 31);
    constexpr int U = kMxAtOnce;                           // groups whose loads are in flight
    // A group of bf16 values that starts anywhere: from the two whole vectors that it lies across (one by one, of 16 bytes apart, 178 us
    // instead of 113 for 65 536 rows of 999 with the pairs of mx_write_values; float32 values one by one are 8 % ahead of vectors).
    constexpr bool kShifted = kRows == kMxAny && sizeof(T) == 2;
    const int64_t vecs = kShifted ? rows * cols / 8 : 0;   // whole ones of the source
    // (whole warps: the shuffles below want all lanes; step is a multiple of 32, and so is the rounded total)
    const int64_t end = (total + 31) & ~(int64_t)31;
    for (int64_t u0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; u0 < end; u0 += U * step) {
        float v[U][8];
        uint4 raw[U][kShifted ? 2 : sizeof(T) / 2];
        int64_t at[U], row[U];
        uint32_t g[U];                                     // group of the row
        int n[U];                                          // elements of the group that exist
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t unit = u0 + u * step;
            row[u] = 0;
            g[u] = 0;
            if (kRows != kMxWhole) row[u] = mx_divide(unit, (uint32_t)(nb * 4), small, g[u]);
            n[u] = unit >= total ? 0 : kRows == kMxWhole ? 8 : (int)max((int64_t)0, min((int64_t)8, cols - (int64_t)g[u] * 8));
            at[u] = kRows == kMxWhole ? unit * 8 : row[u] * cols + (int64_t)g[u] * 8;
            if constexpr (kRows != kMxAny) {
                // (without a branch, which would have the next load wait: a group that does not exist reads the first one)
                const uint4* from = reinterpret_cast<const uint4*>(src + (n[u] ? at[u] : 0));
                raw[u][0] = __ldcs(from);
                if constexpr (sizeof(T) == 4) raw[u][1] = __ldcs(from + 1);
            } else {
                if constexpr (kShifted) {
                    at[u] = min(at[u], rows * cols);       // (groups that do not exist)
                    if (vecs > 0) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) raw[u][k] = __ldg(reinterpret_cast<const uint4*>(src) + min(at[u] / 8 + k, vecs - 1));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[u][e] = load_float(src + (e < n[u] ? at[u] + e : 0));
                }
            }
        }
        if constexpr (kRows == kMxAny) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if constexpr (kShifted) {
                    mx_shift(raw[u], (int)(at[u] & 7), v[u]);
                    if (at[u] + 8 > vecs * 8) {            // what is left behind the last whole vector
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[u][e] = e < n[u] ? load_float(src + at[u] + e) : 0.0f;
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] = e < n[u] ? v[u][e] : 0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t unit = u0 + u * step;
            if (unit - (threadIdx.x & 31) >= total) break;                    // (the same answer in a whole warp)
            unsigned a = 0;                                                   // largest magnitude, as the bits of a float32
            if constexpr (kRows != kMxAny && sizeof(T) == 2) {
                const uint4 w = raw[u][0];
                Elem<T>::unpack(w, v[u]);
                const unsigned two = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
                a = max(two & 0xffff0000u, two << 16);
            } else if constexpr (kRows != kMxAny) {
                const uint32_t w[8] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w, raw[u][1].x, raw[u][1].y, raw[u][1].z, raw[u][1].w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[u][e] = __uint_as_float(w[e]);
                    a = max(a, w[e] & 0x7fffffffu);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) a = max(a, __float_as_uint(v[u][e]) & 0x7fffffffu);
            }
            if (n[u] == 0) a = 0;                                             // (a group that does not exist, in a block that does)
            a = max(a, __shfl_xor_sync(kFullMask, a, 1));
            a = max(a, __shfl_xor_sync(kFullMask, a, 2));
            const int s = mx_block_scale(a);
            // 2^(127 - s): at most 2^127, and products of it are exact but for those far below the smallest code
            const float inv = __uint_as_float((unsigned)max(254 - s, 0) << 23);
            uint32_t word = 0;
#pragma unroll
            for (int e = 0; e < 8; e += 2)
                word |= (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(v[u][e] * inv, v[u][e + 1] * inv), __NV_E2M1, cudaRoundNearest) << (4 * e);
            if (s == 255) word = 0;
            if (n[u] == 0) continue;
            if constexpr (kRows != kMxAny) {
                *reinterpret_cast<uint32_t*>(codes + (kRows == kMxWhole ? unit * 4 : row[u] * cb + (int64_t)g[u] * 4)) = word;
            } else {
                uint8_t* to = codes + row[u] * cb + (int64_t)g[u] * 4;
                if (cb % 4 == 0) {
                    *reinterpret_cast<uint32_t*>(to) = word;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        if (e < n[u]) to[e >> 1] = (uint8_t)(word >> (4 * e));
                }
            }
            if (((kRows == kMxWhole ? (uint32_t)unit : g[u]) & 3) == 0) scales[kRows == kMxWhole ? unit >> 2 : row[u] * nb + (g[u] >> 2)] = (uint8_t)s;
            if (values) mx_write_values(values + at[u], word, s, n[u], kRows == kMxAny ? mx_store_elements(cols) : 8);
        }
    }
}

template <typename T, int kRows>
__global__ void __launch_bounds__(256)
k_dequantize_mx4(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ values, int64_t rows, int64_t cols)
{
    pdl_trigger();
    pdl_wait();
    const int64_t nb = mx_scales(cols), cb = mx_code_bytes(cols), total = rows * nb * 4;
    const int64_t step = (int64_t)gridDim.x * blockDim.x;
    const bool small = total + 4 * step < ((int64_t)1 << 31);
    for (int64_t unit = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; unit < total; unit += step) {
        uint32_t g = 0;
        const int64_t row = kRows == kMxWhole ? 0 : mx_divide(unit, (uint32_t)(nb * 4), small, g);
        const int n = kRows == kMxWhole ? 8 : (int)max((int64_t)0, min((int64_t)8, cols - (int64_t)g * 8));
        if (n == 0) continue;
        uint32_t word = 0;
        if constexpr (kRows != kMxAny) word = __ldcs(reinterpret_cast<const uint32_t*>(codes + (kRows == kMxWhole ? unit * 4 : row * cb + (int64_t)g * 4)));
        else if (cb % 4 == 0) word = __ldcs(reinterpret_cast<const uint32_t*>(codes + row * cb + (int64_t)g * 4));
        else
            for (int e = 0; e < n; e += 2) word |= (uint32_t)codes[row * cb + (int64_t)g * 4 + (e >> 1)] << (4 * e);
        const int sc = __ldg(scales + (kRows == kMxWhole ? unit >> 2 : row * nb + (g >> 2)));
        mx_write_values(values + (kRows == kMxWhole ? unit * 8 : row * cols + (int64_t)g * 8), word, sc, n, kRows == kMxAny ? mx_store_elements(cols) : 8);
    }
}

// ---- images ----------------------------------------------------------------------------------------

// A word of an image holds eight codes so that a shift and a mask put two of them in the sign, low exponent and top mantissa bits of
// the two halves of a register: in each half, code pair 0 at bits 15 and 8..6, pair 1 three and pair 2 six places lower, and pair 3 in
// the four bits that are left (sign 14, magnitude 13, 11 and 10).  Pair p of the word: codes 2p (low half) and 2p + 1.
__host__ __device__ inline uint32_t mx_image_word(const uint32_t (&code)[8]) {
    uint32_t w = 0;
    for (int e = 0; e < 8; ++e) {
        const uint32_t s = code[e] >> 3, m = code[e] & 7u, base = 16u * (e & 1);
        const int p = e >> 1;
        if (p < 3) w |= (s << (15 - 3 * p) | m << (6 - 3 * p)) << base;
        else w |= (s << 14 | (m >> 2) << 13 | (m & 3u) << 10) << base;
    }
    return w;
}

// The four registers of a word, as bf16 values that lack a factor 2^126.
__device__ __forceinline__ void mx_expand(uint32_t w, uint32_t (&r)[4]) {
    constexpr uint32_t kM = 0x81C081C0u;
    r[0] = w & kM;
    r[1] = (w << 3) & kM;
    r[2] = (w << 6) & kM;
    r[3] = ((w << 1) & 0x80008000u) | ((w >> 5) & 0x01000100u) | ((w >> 4) & 0x00C000C0u);
}
// The same for two codes with scales of their own (low byte of lo and of hi).
__device__ __forceinline__ uint32_t mx_pair(uint32_t lo, uint32_t hi) { return (lo & 0xffffu) | (hi & 0xffff0000u); }

constexpr int kMxUnit = 64;            // columns of x per step of the first product, outputs per step of the second

// A layer's image: one record per leaf with everything that its evaluation reads, so that one request brings it: codes of W1, their
// scales, codes of W2, their scales, both biases (bf16).  Leaves of 8 neurons and more (tensor cores): the operands of mma.sync in the
// order in which a warp loads them.  Thinner ones (CUDA cores): rows.  In both a row's columns are padded with zero codes.
struct MxLayout {
    int D, O, l;
    bool mma;
    __host__ __device__ int units1() const { return (D + kMxUnit - 1) / kMxUnit; }
    __host__ __device__ int units2() const { return (O + kMxUnit - 1) / kMxUnit; }
    __host__ __device__ int Kp() const { return l <= 16 ? 16 : (l + 31) / 32 * 32; }      // hidden units as the second product sees them
    // sizes of the parts, then their places in the record, in bytes
    __host__ __device__ int w1() const { return mma ? units1() * l * 32 : l * ((D + 7) / 8) * 4; }
    __host__ __device__ int s1() const { return mma ? units1() * l * 2 : l * (int)mx_scales(D); }
    __host__ __device__ int w2() const { return mma ? units2() * Kp() * 32 : l * ((O + 7) / 8) * 4; }
    __host__ __device__ int s2() const { return mma ? units2() * 2 * Kp() : l * (int)mx_scales(O); }
    __host__ __device__ static int up(int bytes) { return (bytes + 15) & ~15; }
    __host__ __device__ int at_s1() const { return up(w1()); }
    __host__ __device__ int at_w2() const { return at_s1() + up(s1()); }
    __host__ __device__ int at_s2() const { return at_w2() + up(w2()); }
    __host__ __device__ int at_b1() const { return at_s2() + up(s2()); }
    __host__ __device__ int at_b2() const { return at_b1() + up(2 * l); }
    __host__ __device__ int record() const { return (at_b2() + up(2 * O) + 127) & ~127; }
};

__device__ __forceinline__ uint32_t caller_code(const uint8_t* __restrict__ codes, int64_t row, int cols, int c) {
    if (c >= cols) return 0u;
    return (codes[row * mx_code_bytes(cols) + (c >> 1)] >> (4 * (c & 1))) & 15u;
}
__device__ __forceinline__ uint8_t image_scale(const uint8_t* __restrict__ scales, int64_t row, int cols, int c, bool big) {
    const int s = c < cols ? scales[row * mx_scales(cols) + c / kMxBlock] : 0;
    return (uint8_t)(big ? s : s + 126);
}

// *big = 1 if a scale is over 2.
__global__ void k_mx_find_big(const uint8_t* __restrict__ scales, int64_t n, int* __restrict__ big)
{
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x)
        if (scales[i] > 128) *big = 1;
}

// w1: caller's codes [leaves * l, D]; w2: [leaves * l, O].
__global__ void k_pack_mx4(const uint8_t* __restrict__ w1, const uint8_t* __restrict__ sc1, const uint8_t* __restrict__ w2,
                           const uint8_t* __restrict__ sc2, const uint16_t* __restrict__ b1, const uint16_t* __restrict__ b2,
                           unsigned char* __restrict__ img, MxLayout L, int64_t n_leaves, bool big)
{
    const int64_t i0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
    const int l = L.l, D = L.D, O = L.O, Kp = L.Kp();
    const int64_t record = L.record();
    auto word_of = [&](const uint8_t* codes, int64_t row, int cols, int c0) {
        uint32_t c[8];
        for (int e = 0; e < 8; ++e) c[e] = caller_code(codes, row, cols, c0 + e);
        return mx_image_word(c);
    };
    // n words (or bytes) per leaf from offset `at` on: k of leaf j is value(j, k)
    auto words = [&](int at, int n, auto&& value) {
        for (int64_t i = i0; i < n_leaves * n; i += step) {
            const int64_t leaf = i / n;
            reinterpret_cast<uint32_t*>(img + leaf * record + at)[i - leaf * n] = value(leaf, (int)(i - leaf * n));
        }
    };
    auto bytes = [&](int at, int n, auto&& value) {
        for (int64_t i = i0; i < n_leaves * n; i += step) {
            const int64_t leaf = i / n;
            (img + leaf * record + at)[i - leaf * n] = value(leaf, (int)(i - leaf * n));
        }
    };
    for (int64_t i = i0; i < n_leaves * l; i += step) reinterpret_cast<uint16_t*>(img + i / l * record + L.at_b1())[i % l] = b1[i];
    for (int64_t i = i0; i < n_leaves * O; i += step) reinterpret_cast<uint16_t*>(img + i / O * record + L.at_b2())[i % O] = b2[i];
    if (!L.mma) {
        const int wd = (D + 7) / 8, wo = (O + 7) / 8, nd = (int)mx_scales(D), no = (int)mx_scales(O);
        words(0, l * wd, [&](int64_t leaf, int k) { return word_of(w1, leaf * l + k / wd, D, k % wd * 8); });
        words(L.at_w2(), l * wo, [&](int64_t leaf, int k) { return word_of(w2, leaf * l + k / wo, O, k % wo * 8); });
        bytes(L.at_s1(), l * nd, [&](int64_t leaf, int k) { return image_scale(sc1, leaf * l + k / nd, D, k % nd * kMxBlock, big); });
        bytes(L.at_s2(), l * no, [&](int64_t leaf, int k) { return image_scale(sc2, leaf * l + k / no, O, k % no * kMxBlock, big); });
        return;
    }
    // W1: [unit of 64 columns][row][quarter of the unit][2 words]; scales [unit][row][half of the unit]
    words(0, L.w1() / 4, [&](int64_t leaf, int k) { return word_of(w1, leaf * l + k % (l * 8) / 8, D, k / (l * 8) * kMxUnit + (k & 7) * 8); });
    bytes(L.at_s1(), L.s1(), [&](int64_t leaf, int k) {
        return image_scale(sc1, leaf * l + k % (l * 2) / 2, D, k / (l * 2) * kMxUnit + (k & 1) * kMxBlock, big);
    });
    // W2: [unit of 64 outputs][block of 32 hidden units][half of the 8 words][lane][4 words], word 2i + r: the hidden units 8c.. of output
    // 8g + 2i + r, lane = (g, c); with 16 hidden units [unit][lane][4 words], word i: units 4c.. of outputs 8g + 2i, then of 8g + 2i + 1.
    words(L.at_w2(), L.w2() / 4, [&](int64_t leaf, int k) {
        const int u = k / (Kp * 8), in = k % (Kp * 8), j = in & 3, lane = (in >> 2) & 31, g = lane >> 2, c = lane & 3;
        uint32_t code[8];
        for (int e = 0; e < 8; ++e) {
            const int word = Kp == 16 ? 2 * j + (e >> 2) : ((in >> 7) & 1) * 4 + j;
            const int unit = Kp == 16 ? 4 * c + (e & 3) : (in >> 8) * 32 + 8 * c + e;
            code[e] = unit < l ? caller_code(w2, leaf * l + unit, O, u * kMxUnit + 8 * g + word) : 0u;
        }
        return mx_image_word(code);
    });
    // scales [unit][half of its outputs][hidden unit]
    bytes(L.at_s2(), L.s2(), [&](int64_t leaf, int k) {
        const int u = k / (2 * Kp), unit = k % Kp;
        return unit < l ? image_scale(sc2, leaf * l + unit, O, u * kMxUnit + k / Kp % 2 * kMxBlock, big) : (uint8_t)(big ? 0 : 126);
    });
}

// ---- leaves on tensor cores ------------------------------------------------------------------------

struct MxLeafArgs {
    const __nv_bfloat16* x;
    const int32_t* perm;               // tokens in bucket order, or the table of lists [n_leaves][cap]
    const Tile* tiles;                 // (counts == nullptr) tile list
    int n_tiles;
    int32_t* counts;                   // entries of every list, [1] CTAs that have finished; zeroed at the end
    int n_leaves, cap;
    const unsigned char* image;        // records of the leaves
    __nv_bfloat16* y;
    MxLayout lay;
    int act, tile_rows;                // tile_rows: a multiple of 8, at most 8 kMxMaxGroups
    bool y_vec;                        // rows of y are 16-byte vectors
    int* status;
};

// 8 consecutive outputs.
__device__ __forceinline__ void mx_store8(__nv_bfloat16* __restrict__ p, int n, bool vec, const uint32_t (&r)[4]) {
    if (vec) {
        if (n > 0) __stcs(reinterpret_cast<uint4*>(p), make_uint4(r[0], r[1], r[2], r[3]));
    } else {
        uint16_t* q = reinterpret_cast<uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (2 * i < n) q[2 * i] = (uint16_t)r[i];
            if (2 * i + 1 < n) q[2 * i + 1] = (uint16_t)(r[i] >> 16);
        }
    }
}
// Sends for [p, p + bytes) into L2 (16-byte aligned, whole 16-byte units).
__device__ __forceinline__ void mx_prefetch(const void* p, int64_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"((uint32_t)bytes) : "memory");
}

constexpr int kMxWarps = 8;
constexpr int kMxThreads = kMxWarps * 32;
constexpr int kMxMaxGroups = 8;              // groups of 8 tokens per tile, at most
constexpr int kMxChunk = 1024;               // columns of x in shared memory at a time, at most

// Shared memory of k_leaf_mx4: token rows (at a pitch of 16 bytes past whole 128-byte lines: the operand loads of 8 rows then touch
// every bank once), partial sums of the first product, hidden values (two bf16 planes), the tokens of this tile and the next, and the
// number of tiles before every leaf and the rows of its last one where tiles come from lists.
struct MxLeafSmem {
    int rows, D, Kp, listed;
    __host__ __device__ int chunk() const { return D < kMxChunk ? (D + kMxUnit - 1) / kMxUnit * kMxUnit : kMxChunk; }
    __host__ __device__ int pitch() const { return chunk() * 2 + 16; }
    __host__ __device__ int x() const { return rows * pitch(); }
    __host__ __device__ int red() const { return kMxWarps * (rows / 8) * 512; }
    __host__ __device__ int hid() const { return rows * Kp * 4; }
    __host__ __device__ int bytes() const { return x() + red() + hid() + 2 * rows * 4 + (listed ? (listed + 1) * 2 + listed + 2 : 0); }
};

// The operand registers of one word of W1 (16 columns: two words), scaled.
template <bool kBig>
__device__ __forceinline__ void mx_row16(uint2 code, uint32_t sc, uint32_t (&r)[8]) {
    uint32_t lo[4], hi[4];
    mx_expand(code.x, lo);
    mx_expand(code.y, hi);
    const uint32_t f1 = mx_mul1(sc, kBig), f2 = kBig ? mx_mul2(sc) : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[i] = mul_bf16x2(lo[i], f1);
        r[4 + i] = mul_bf16x2(hi[i], f1);
        if (kBig) { r[i] = mul_bf16x2(r[i], f2); r[4 + i] = mul_bf16x2(r[4 + i], f2); }
    }
}

// A warp's share of the first product for 16 hidden units and all tokens of the tile, over the columns in shared memory.  Weights are
// the MMAs' 16 rows, tokens their 8 columns.  The order of the summands is free, so lane c of a quad takes 16 consecutive columns (32
// bytes of a token's row, 8 of codes, one scale) for four MMAs.  Codes go from global memory straight into the operands, kMxAhead steps
// ahead (all of a warp's steps for up to 1024 columns), the first of them sent for before the tokens are waited for.
constexpr int kMxAhead = 4;
struct MxCodes {
    uint2 code[kMxAhead][2];
    uint32_t sc[kMxAhead][2];
};
// (Rows past the leaf's last repeat it: their sums are not used.  u past the last unit likewise.)
__device__ __forceinline__ void mx_fetch_codes(const unsigned char* __restrict__ rec, int at_s1, int l, int row0, int u, int u1, int lane, MxCodes& q, int k) {
    const int g = lane >> 2, c = lane & 3;
    const int base = min(u, u1 - 1) * l;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = base + min(row0 + 8 * h + g, l - 1);
        q.code[k][h] = __ldg(reinterpret_cast<const uint2*>(rec) + row * 4 + c);
        q.sc[k][h] = __ldg(rec + at_s1 + row * 2 + (c >> 1));
    }
}
template <bool kBig, int G>
__device__ __forceinline__ void mx_hidden(const unsigned char* __restrict__ rec, int at_s1, int l, MxCodes& q, const unsigned char* xs, int pitch,
                                          int groups, int row0, int u0, int u1, int step, int unit_base, int lane, float (&acc)[G][4])
{
    const int g = lane >> 2, c = lane & 3;
    for (int u = u0; u < u1; u += kMxAhead * step) {
#pragma unroll
        for (int k = 0; k < kMxAhead; ++k) {
            const int uk = u + k * step;
            if (uk >= u1) break;
            uint32_t w[2][8];
#pragma unroll
            for (int h = 0; h < 2; ++h) mx_row16<kBig>(q.code[k][h], q.sc[k][h], w[h]);
            if (uk + kMxAhead * step < u1) mx_fetch_codes(rec, at_s1, l, row0, uk + kMxAhead * step, u1, lane, q, k);
            const unsigned char* xp = xs + g * pitch + (uk - unit_base) * (kMxUnit * 2) + 32 * c;
            // (two groups at a time, whose MMAs do not wait for one another; a last odd group is computed twice)
#pragma unroll
            for (int t = 0; t < G; t += 2) {
                if (t >= groups) break;
                const unsigned char *xa = xp + t * 8 * pitch, *xb = t + 1 < groups ? xa + 8 * pitch : xa;
                const uint4 a0 = *reinterpret_cast<const uint4*>(xa), b0 = *reinterpret_cast<const uint4*>(xb);
                const uint4 a1 = *reinterpret_cast<const uint4*>(xa + 16), b1 = *reinterpret_cast<const uint4*>(xb + 16);
                ptx::mma_bf16(acc[t], w[0][0], w[1][0], w[0][1], w[1][1], a0.x, a0.y);
                ptx::mma_bf16(acc[t + 1], w[0][0], w[1][0], w[0][1], w[1][1], b0.x, b0.y);
                ptx::mma_bf16(acc[t], w[0][2], w[1][2], w[0][3], w[1][3], a0.z, a0.w);
                ptx::mma_bf16(acc[t + 1], w[0][2], w[1][2], w[0][3], w[1][3], b0.z, b0.w);
                ptx::mma_bf16(acc[t], w[0][4], w[1][4], w[0][5], w[1][5], a1.x, a1.y);
                ptx::mma_bf16(acc[t + 1], w[0][4], w[1][4], w[0][5], w[1][5], b1.x, b1.y);
                ptx::mma_bf16(acc[t], w[0][6], w[1][6], w[0][7], w[1][7], a1.z, a1.w);
                ptx::mma_bf16(acc[t + 1], w[0][6], w[1][6], w[0][7], w[1][7], b1.z, b1.w);
            }
        }
    }
}

// The raw operands of a K-block of 64 outputs, and the outputs' biases.
struct MxNext {
    uint4 q0, q1, bias;
    uint2 sc;
};
template <bool K16>
__device__ __forceinline__ void mx_fetch_outputs(const MxLayout& Ly, const unsigned char* __restrict__ rec, int u, int kb, int lane, MxNext& next) {
    if (u >= Ly.units2()) return;
    const int g = lane >> 2, c = lane & 3, Kp = K16 ? 16 : Ly.Kp();
    const uint4* src = reinterpret_cast<const uint4*>(rec + Ly.at_w2()) + (K16 ? u * 32 : (u * (Kp / 32) + kb) * 64) + lane;
    const unsigned char* sp = rec + Ly.at_s2() + (u * 2 + (g >> 2)) * Kp + kb * 32 + (K16 ? 4 : 8) * c;
    next.q0 = __ldg(src);
    if constexpr (K16) {
        next.sc.x = __ldg(reinterpret_cast<const uint32_t*>(sp));
    } else {
        next.q1 = __ldg(src + 32);
        next.sc = __ldg(reinterpret_cast<const uint2*>(sp));
    }
    if (kb == 0 && u * kMxUnit + 8 * g < Ly.O)             // (to the end of 16 bytes: records are padded)
        next.bias = __ldg(reinterpret_cast<const uint4*>(rec + Ly.at_b2()) + u * 8 + g);
}

// The second product: units u0, u0 + step, .. of 64 outputs for all tokens of a tile, by one warp; numbered so that a lane ends with 8
// consecutive outputs of its tokens and 8 lanes with 128 bytes of a row.  hid: hidden values [2][R][Kp] (the two summands of each);
// next: the operands of (u0, 0), fetched before.  TG token groups at a time: their MMAs do not wait for one another (a last odd group is
// computed twice), and wider leaves expand every K-block once for all of them.
template <bool K16, bool kWide, bool kBig, int TG>
__device__ __forceinline__ void mx_outputs(__nv_bfloat16* __restrict__ y, bool y_vec, const MxLayout& Ly, const unsigned char* __restrict__ rec,
                                           const __nv_bfloat16* hid, int R, int rows, const int* s_tok, int u0, int step, int lane, MxNext& next)
{
    constexpr int P = K16 ? 2 : 4;
    const int g = lane >> 2, c = lane & 3, O = Ly.O, units2 = Ly.units2(), Kp = K16 ? 16 : kWide ? Ly.Kp() : 32, kblocks = kWide ? Kp / 32 : 1;
    const int groups = (rows + 7) / 8;
    auto fetch = [&](int u, int kb) { mx_fetch_outputs<K16>(Ly, rec, u, kb, lane, next); };
    for (int u = u0; u < units2; u += step) {
        const int o = u * kMxUnit + 8 * g, n = O - o;
        // biases as the sums that the MMAs start from: outputs 2 i and 2 i + 1 of two tokens
        float bias[4][4];
        {
            const uint32_t bw[4] = {next.bias.x, next.bias.y, next.bias.z, next.bias.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bias[i][0] = bias[i][1] = __uint_as_float(bw[i] << 16);
                bias[i][2] = bias[i][3] = __uint_as_float(bw[i] & 0xffff0000u);
            }
        }
        uint32_t w[8][P];                              // [2 i + row][pair of hidden units]
        bool infinite = false;                         // (kBig) some of them may be: scales of 2^126 and more
        auto operands = [&]() {
            if constexpr (kBig) {
                unsigned huge = __vcmpgeu4(next.sc.x, 0xfdfdfdfdu);
                if constexpr (!K16) huge |= __vcmpgeu4(next.sc.y, 0xfdfdfdfdu);
                infinite = __any_sync(kFullMask, huge);
            }
            uint32_t f1[P], f2[P];                     // the scales of a pair of hidden units are neighbouring bytes
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const uint32_t two = p < 2 ? next.sc.x : next.sc.y, lo = (two >> (16 * (p & 1))) & 0xffu, hi = (two >> (16 * (p & 1) + 8)) & 0xffu;
                f1[p] = mx_pair(mx_mul1(lo, kBig), mx_mul1(hi, kBig));
                f2[p] = kBig ? mx_pair(mx_mul2(lo), mx_mul2(hi)) : 0u;
            }
            const uint32_t q[8] = {next.q0.x, next.q0.y, next.q0.z, next.q0.w, next.q1.x, next.q1.y, next.q1.z, next.q1.w};
#pragma unroll
            for (int i = 0; i < (K16 ? 4 : 8); ++i) {
                uint32_t r[4];
                mx_expand(q[i], r);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int row = K16 ? 2 * i + (k >> 1) : i, p = K16 ? k & 1 : k;
                    w[row][p] = mul_bf16x2(r[k], f1[p]);
                    if (kBig) w[row][p] = mul_bf16x2(w[row][p], f2[p]);
                }
            }
        };
        if (!kWide) {
            operands();
            fetch(u + step, 0);
        }
        for (int t0 = 0; t0 < groups; t0 += TG) {
            float acc[TG][4][4];
            const __nv_bfloat16* h[TG];
#pragma unroll
            for (int t = 0; t < TG; ++t) {
                h[t] = hid + (8 * (t0 + t < groups ? t0 + t : t0) + g) * Kp + (K16 ? 4 : 8) * c;
                if constexpr (kWide) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[t][i][k] = bias[i][k];
                }
            }
            // outputs 2 i and 2 i + 1 of every token group, from pair `pair` of the hidden units on; the first to come takes the biases
            auto multiply = [&](int pair, const uint32_t (&b)[TG][2], bool first) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int t = 0; t < TG; ++t) {
                        if (first) ptx::mma_bf16_from(acc[t][i], bias[i], w[2 * i][pair], w[2 * i + 1][pair], w[2 * i][pair + 1], w[2 * i + 1][pair + 1], b[t][0], b[t][1]);
                        else ptx::mma_bf16(acc[t][i], w[2 * i][pair], w[2 * i + 1][pair], w[2 * i][pair + 1], w[2 * i + 1][pair + 1], b[t][0], b[t][1]);
                    }
            };
            // The same without weights that are no numbers, for the second summand of the hidden values: an infinite weight times the first
            // is the product, and one of the second, of the other sign or zero, would make a NaN of it.
            auto multiply_finite = [&](int pair, const uint32_t (&b)[TG][2]) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t f[4] = {mx_finite(w[2 * i][pair]), mx_finite(w[2 * i + 1][pair]), mx_finite(w[2 * i][pair + 1]), mx_finite(w[2 * i + 1][pair + 1])};
#pragma unroll
                    for (int t = 0; t < TG; ++t) ptx::mma_bf16(acc[t][i], f[0], f[1], f[2], f[3], b[t][0], b[t][1]);
                }
            };
            for (int kb = 0; kb < kblocks; ++kb) {
                if (kWide) {
                    operands();
                    if (kb + 1 < kblocks) fetch(u, kb + 1);
                    else fetch(t0 + TG < groups ? u : u + step, 0);
                }
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    uint32_t b[2][TG][2];
#pragma unroll
                    for (int t = 0; t < TG; ++t) {
                        const __nv_bfloat16* from = h[t] + p * R * Kp + kb * 32;
                        if constexpr (K16) {
                            const uint2 q = *reinterpret_cast<const uint2*>(from);
                            b[0][t][0] = q.x; b[0][t][1] = q.y;
                        } else {
                            const uint4 q = *reinterpret_cast<const uint4*>(from);
                            b[0][t][0] = q.x; b[0][t][1] = q.y; b[1][t][0] = q.z; b[1][t][1] = q.w;
                        }
                    }
                    if (kBig && p == 1 && infinite) {
                        multiply_finite(0, b[0]);
                        if constexpr (!K16) multiply_finite(2, b[1]);
                        continue;
                    }
                    multiply(0, b[0], !kWide && p == 0);
                    if constexpr (!K16) multiply(2, b[1], false);
                }
            }
#pragma unroll
            for (int t = 0; t < TG; ++t) {
                if (t0 + t >= groups) break;
                const int2 tok = *reinterpret_cast<const int2*>(s_tok + 8 * (t0 + t) + 2 * c);
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int to = r ? tok.y : tok.x;
                    uint32_t out[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) out[i] = ptx::pack_bf16(acc[t][i][r], acc[t][i][2 + r]);
                    if (8 * (t0 + t) + 2 * c + r < rows) mx_store8(y + (int64_t)to * O + o, n, y_vec, out);
                }
            }
        }
    }
}

// The bin that tile idx belongs to: the last b with pre[b] <= idx.  By a whole warp: 32 places at a time.
__device__ __forceinline__ int mx_bin_of_tile(const uint16_t* pre, int n_bins, int idx, int lane) {
    int lo = 0, n = n_bins;                                // in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const unsigned at_or_before = __ballot_sync(kFullMask, lane * step < n && pre[at] <= idx);
        const int k = 31 - __clz(at_or_before);            // (pre is sorted and pre[lo] <= idx)
        n = min(step, n - k * step);
        lo += k * step;
    }
    return lo;
}

// Rows of bf16 values from one length to another, the vectors of the leaf kernels from and to rows that start anywhere: whole vectors are
// stored, each put together from the two of the source that it lies across, by a shift that is the same in a row.  A warp per row, of up
// to eight vectors four rows.  Bound: HBM (65 536 rows of 1023: 64 us to whole vectors, 87 from them; floor 41).
__global__ void __launch_bounds__(256)
k_mx4_copy_rows(uint16_t* __restrict__ dst, int dst_cols, const uint16_t* __restrict__ src, int src_cols, int64_t rows)
{
    const int span = dst_cols <= 64 ? 8 : 32, lane = threadIdx.x & (span - 1), cols = min(dst_cols, src_cols), at_once = blockDim.x / span;
    const uint16_t* end = src + rows * src_cols;
    pdl_trigger();
    pdl_wait();
    for (int64_t row = (int64_t)blockIdx.x * at_once + threadIdx.x / span; row < rows; row += (int64_t)gridDim.x * at_once) {
        const uint16_t* s = src + row * src_cols;
        uint16_t* d = dst + row * dst_cols;
        const int j0 = min(dst_cols, (int)(-(reinterpret_cast<uintptr_t>(d) >> 1) & 7)), vecs = (dst_cols - j0) >> 3;
        const int sh = (int)((reinterpret_cast<uintptr_t>(s + j0) >> 1) & 7);          // elements of a vector before the first wanted
        const bool inside = s + cols + 8 <= end;                             // no vector reaches past the buffer
#pragma unroll 4
        for (int i = lane; i < vecs; i += span) {
            const int j = j0 + 8 * i;
            const uint16_t* from = s + j - sh;                               // (on or behind the buffer's start, which is on such a boundary)
            uint32_t w[9];
            if (inside) {
                // (without branches: the second vector, or the first again)
                const uint4 a = __ldg(reinterpret_cast<const uint4*>(from));
                const uint4 b = __ldg(reinterpret_cast<const uint4*>(sh > 0 && j + 8 - sh < cols ? from + 8 : from));
                w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t lo = from + 2 * k < end ? from[2 * k] : 0, hi = from + 2 * k + 1 < end ? from[2 * k + 1] : 0;
                    w[k] = lo | hi << 16;
                }
            }
            w[8] = 0;
            if (sh & 4) {
#pragma unroll
                for (int k = 0; k < 6; ++k) w[k] = w[k + 2];
            }
            if (sh & 2) {
#pragma unroll
                for (int k = 0; k < 5; ++k) w[k] = w[k + 1];
            }
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                o[k] = sh & 1 ? __funnelshift_r(w[k], w[k + 1], 16) : w[k];
                const int left = cols - (j + 2 * k);                         // wanted of these two
                o[k] = left >= 2 ? o[k] : left == 1 ? o[k] & 0xffffu : 0u;
            }
            *reinterpret_cast<uint4*>(d + j) = make_uint4(o[0], o[1], o[2], o[3]);
        }
        const int rest = j0 + 8 * vecs;
        if (lane < j0) d[lane] = lane < cols ? s[lane] : (uint16_t)0;
        if (lane < 8 && rest + lane < dst_cols) d[rest + lane] = rest + lane < cols ? s[rest + lane] : (uint16_t)0;
    }
}

// A CTA per tile of up to tile_rows tokens of one leaf, two CTAs per SM.  Token rows come by bulk copies; those of the next tile are
// sent for as soon as this tile's first product is done with the buffer, and arrive while its hidden values and outputs are computed;
// the next leaf's record is sent for to L2 at the same time.  The first product is split along D over the warps (MT = 2: over the two
// groups of 16 hidden units too), so that no weight is expanded twice; the sums meet in shared memory, where bias and activation are
// applied; for the second product every warp has output columns of its own.  Hidden values are kept as sums of two bf16 values (float32 precision to 2^-16):
// the extra MMAs cost little next to the expansion.  Bound: latency and issue slots (42 % busy) with the 16 warps that 128 registers allow (leaves
// of 17 to 32 spill 96 bytes there, the others 8); 1024 -> 1024, 2048 leaves of 32, 65 536 tokens 112 us, where its bytes take 46; more warps spill
// more, fewer rows per tile expand weights twice.  The kernels that expand nothing are ahead: the whole forward takes 180 to 186 us there and 165
// to 174 with bf16 weights, 66 and 61 to 63 on 768 -> 768, 256 leaves of 12, 50 432 tokens.
// kWide, the latter with 48, 64 and 96 neurons per leaf: 102, 103 and 166 us (forward 124, 125 and 188; bf16 71, 76 and, on CUDA cores, 835);
// 512 -> 512, 64 leaves of 256: 258 us (290; 1239).
// MT: groups of 16 hidden units at a time: 1 for leaves of up to 16 (one K-block of 16 in the second product), else 2.
// kWide: more than 32 hidden units: several passes over x, several K-blocks in the second product.
template <int MT, bool kWide, bool kBig>
__global__ void __launch_bounds__(kMxThreads, 2)
k_leaf_mx4(const MxLeafArgs A)
{
    static_assert(!kWide || MT == 2, "leaves of up to 16 have one K-block");
    constexpr bool K16 = MT == 1;
    constexpr int NW = kMxWarps, kThreads = kMxThreads;
    constexpr int kSplit = NW / MT;                        // warps that share a group of 16 hidden units
    extern __shared__ __align__(16) unsigned char smem_mx[];
    __shared__ int s_wsum[NW], s_last, s_next[2][3];       // s_next: tile, leaf, rows
    __shared__ uint64_t s_full;
    const MxLayout& Ly = A.lay;
    const int l = Ly.l, D = Ly.D, Kp = K16 ? 16 : kWide ? Ly.Kp() : 32;
    const int R = A.tile_rows;
    const MxLeafSmem S{R, D, Kp, A.counts ? A.n_leaves : 0};
    unsigned char* xs = smem_mx;
    float* red = reinterpret_cast<float*>(smem_mx + S.x());                           // [warp][token group][register][lane]
    __nv_bfloat16* hid = reinterpret_cast<__nv_bfloat16*>(smem_mx + S.x() + S.red()); // [2][R][Kp]
    int* s_tok2 = reinterpret_cast<int*>(smem_mx + S.x() + S.red() + S.hid());        // [2][R]
    uint16_t* s_pre = reinterpret_cast<uint16_t*>(s_tok2 + 2 * R);                    // [n_leaves + 1]
    uint8_t* s_rest = reinterpret_cast<uint8_t*>(s_pre + A.n_leaves + 1);             // [n_leaves]
    const int pitch = S.pitch(), chunk = S.chunk(), chunks = (D + chunk - 1) / chunk;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    if (tid == 0) {
        ptx::mbar_init(&s_full, 1);
        ptx::fence_mbar_init();
    }
    // columns past D stay zero: the copies do not touch them
    for (int i = tid; i < S.x() / 16; i += kThreads) reinterpret_cast<uint4*>(xs)[i] = make_uint4(0u, 0u, 0u, 0u);
    ptx::fence_proxy_async();
    pdl_trigger();
    __syncthreads();
    pdl_wait();
    if (A.counts)
        tiles_before_bins([&](int b) {
            const int n = __ldcg(A.counts + b);
            s_rest[b] = (uint8_t)((n + R - 1) % R + 1);
            return n;
        }, A.n_leaves, R, s_pre, s_wsum, kThreads);
    const int n_tiles = A.counts ? s_pre[A.n_leaves] : A.n_tiles;
    const int units1 = Ly.units1(), at_s1 = Ly.at_s1(), at_b1 = Ly.at_b1();
    const int64_t record = Ly.record();

    // The first tile from `tile` on that is not empty (a list of tiles may contain empty ones); rows = 0: none.  Tokens `lane` and
    // `lane + 32` of it in tok.  By a whole warp.
    struct Found { int tile, leaf, rows, tok[2]; };
    auto find_tile = [&](int tile) {
        Found f;
        f.tile = n_tiles;
        f.leaf = f.rows = 0;
        f.tok[0] = f.tok[1] = -1;
        const int32_t* list = nullptr;
        if (A.counts) {
            if (tile < n_tiles) {
                f.tile = tile;
                f.leaf = mx_bin_of_tile(s_pre, A.n_leaves, tile, lane);
                f.rows = tile + 1 < s_pre[f.leaf + 1] ? R : s_rest[f.leaf];
                list = A.perm + (int64_t)f.leaf * A.cap + (tile - s_pre[f.leaf]) * R;
            }
        } else {
            for (; tile < n_tiles; tile += 32 * gridDim.x) {
                const int64_t mine = tile + (int64_t)lane * gridDim.x;
                Tile t;
                t.rows = 0;
                if (mine < n_tiles) t = A.tiles[mine];
                const unsigned some = __ballot_sync(kFullMask, t.rows > 0);
                if (some) {
                    const int k = __ffs(some) - 1;
                    f.tile = tile + k * gridDim.x;
                    f.leaf = __shfl_sync(kFullMask, t.bin, k);
                    f.rows = __shfl_sync(kFullMask, t.rows, k);
                    list = A.perm + __shfl_sync(kFullMask, t.start, k);
                    break;
                }
            }
        }
        if (lane < f.rows) f.tok[0] = __ldcg(list + lane);
        if (lane + 32 < f.rows) f.tok[1] = __ldcg(list + lane + 32);
        return f;
    };
    // sends for columns [k0, k0 + chunk) of a tile's rows
    auto send_x = [&](const Found& f, int k0) {
        const int bytes = min(chunk, D - k0) * 2;
        if (lane == 0) ptx::mbar_arrive_expect_tx(&s_full, (uint32_t)(bytes * f.rows));
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (f.tok[h] >= 0) ptx::bulk_g2s(xs + (lane + 32 * h) * pitch, A.x + (int64_t)f.tok[h] * D + k0, (uint32_t)bytes, &s_full);
    };
    auto announce = [&](const Found& f, int buf) {
        if (lane < R) s_tok2[buf * R + lane] = f.tok[0];
        if (lane + 32 < R) s_tok2[buf * R + lane + 32] = f.tok[1];
        if (lane == 0) { s_next[buf][0] = f.tile; s_next[buf][1] = f.leaf; s_next[buf][2] = f.rows; }
        if (f.rows > 0) {
            send_x(f, 0);
            if (lane == 0) mx_prefetch(A.image + f.leaf * record, record);
        }
    };
    // The last warp (which has the least to do where units do not come out even) finds the tiles and sends for their rows.
    constexpr int kFinder = NW - 1;
    Found mine, following;
    if (warp == kFinder) {
        mine = find_tile(blockIdx.x);
        announce(mine, 0);
    }
    __syncthreads();
    uint32_t phase = 0;
    bool timed_out = false;
    // which part of the sums this warp puts together: unit group, register, first token group
    const int my_m = MT == 1 ? 0 : warp >> 2, my_i = warp & 3, my_t = MT == 1 ? warp >> 2 : 0;

    // Two barriers per tile: one between the partial sums and the hidden values, one between those and the outputs.  A warp that has
    // written its outputs goes on to the next tile, which the finder announced between the two (sums, hidden values, tokens and the
    // announcement are not written again before every warp has passed the first barrier of that tile).
    for (int buf = 0;; buf ^= 1) {
        const int tile = s_next[buf][0], leaf = s_next[buf][1], rows = s_next[buf][2];
        if (tile >= n_tiles) break;
        const int groups = (rows + 7) / 8;
        const int* s_tok = s_tok2 + buf * R;
        const unsigned char* rec = A.image + leaf * record;
        if (warp == kFinder) following = find_tile(tile + gridDim.x);

        MxNext next;

        // ---- hidden values
        for (int unit0 = 0; unit0 < l; unit0 += 16 * MT) {
            const bool last_pass = !kWide || unit0 + 16 * MT >= l;
            const int my_unit = unit0 + 16 * my_m + g + 8 * (my_i >> 1);
            const float my_bias = my_unit < l ? __bfloat162float(__ldg(reinterpret_cast<const __nv_bfloat16*>(rec + at_b1) + my_unit)) : 0.0f;
            float acc[kMxMaxGroups][4];
#pragma unroll
            for (int t = 0; t < kMxMaxGroups; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][i] = 0.0f;
            for (int ch = 0; ch < chunks; ++ch) {
                const int k0 = ch * chunk, ub = k0 / kMxUnit, u0 = ub + warp % kSplit, u1 = min(units1, ub + chunk / kMxUnit);
                const int row0 = unit0 + 16 * (warp / kSplit);
                MxCodes q;
#pragma unroll
                for (int k = 0; k < kMxAhead; ++k) mx_fetch_codes(rec, at_s1, l, row0, u0 + k * kSplit, u1, lane, q, k);
                const bool fresh = unit0 == 0 || chunks > 1;           // (one chunk stays for all passes)
                if (ch > 0 || (unit0 > 0 && chunks > 1)) {             // (the first chunk of the first pass is on its way)
                    __syncthreads();
                    if (warp == kFinder) send_x(mine, k0);
                }
                if (fresh) {
                    if (!timed_out && !ptx::mbar_wait_suspended(&s_full, phase)) timed_out = true;
                    phase ^= 1;
                }
                const int past = min(chunk, (units1 - ub) * kMxUnit);      // columns that the MMAs read
                if (chunks > 1 && k0 + past > D) {
                    // the last chunk's columns past D hold an earlier chunk's, which zero codes do not undo where they are infinite
                    for (int r = warp; r < rows; r += NW)
                        for (int k = D - k0 + lane; k < past; k += 32) reinterpret_cast<__nv_bfloat16*>(xs + r * pitch)[k] = __float2bfloat16_rn(0.0f);
                    ptx::fence_proxy_async();              // (the next copies write there)
                    __syncthreads();
                }
                mx_hidden<kBig, kMxMaxGroups>(rec, at_s1, l, q, xs, pitch, groups, row0, u0, u1, kSplit, ub, lane, acc);
            }
#pragma unroll
            for (int t = 0; t < kMxMaxGroups; ++t) {
                if (t >= groups) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) red[((warp * groups + t) * 4 + i) * 32 + lane] = acc[t][i];
            }
            __syncthreads();
            if (last_pass) {
                if (warp == kFinder) announce(following, buf ^ 1);
                mx_fetch_outputs<K16>(Ly, rec, warp, 0, lane, next);
            }
            with_activation(A.act, [&](auto act) {
                const float* from = red + (my_m * kSplit * groups * 4 + my_i) * 32 + lane;
                __nv_bfloat16* to = hid + (2 * c + (my_i & 1)) * Kp + my_unit;
#pragma unroll 2
                for (int t = my_t; t < groups; t += MT == 1 ? 2 : 1) {
                    float sum = my_bias;
#pragma unroll
                    for (int w = 0; w < kSplit; ++w) sum += from[(w * groups + t) * 128];
                    float h = activate_bf16(decltype(act)::value, sum);
                    if (my_unit >= l) h = 0.0f;
                    const __nv_bfloat16 hi = __float2bfloat16_rn(h);
                    const float f = __bfloat162float(hi);
                    to[8 * t * Kp] = hi;
                    to[(R + 8 * t) * Kp] = __float2bfloat16_rn(isinf(f) ? 0.0f : h - f);
                }
            });
            __syncthreads();
        }

        // ---- outputs
        mx_outputs<K16, kWide, kBig, 2>(A.y, A.y_vec, Ly, rec, hid, R, rows, s_tok, warp, NW, lane, next);
        mine = following;
    }
    if (timed_out) {
        if (lane == 0) atomicExch(A.status, kDevTimeout);
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);     // let bulk copies still in flight land before exit
    }
    // the last CTA to finish clears the counts (and the word behind them that counts the CTAs) for the next call
    if (A.counts) {
        __syncthreads();
        if (tid == 0) {
            __threadfence();
            s_last = atomicAdd(A.counts + A.n_leaves, 1) == (int)gridDim.x - 1 ? 1 : 0;
        }
        __syncthreads();
        if (s_last)
            for (int b = tid; b <= A.n_leaves; b += kThreads) A.counts[b] = 0;
    }
}

// ---- a few tokens ----------------------------------------------------------------------------------

struct MxTokenArgs {
    const __nv_bfloat16 *x, *node_w, *node_b;
    const unsigned char* image;
    __nv_bfloat16* y;
    int32_t *leaf_out, *leaf_out2;     // (leaf_out2 may be nullptr)
    MxLayout lay;
    int depth, act;
    int x_cols;                        // row length of x: D, or less where D is rounded up
    bool y_vec, big;                   // rows of y are 16-byte vectors; (k_mx4_token_rows) some scale is over 2
};

// Shared memory: the token's row padded with zeros, partial sums, hidden values (eight rows of them: the operand of an MMA).
struct MxTokenSmem {
    int D, Kp;
    __host__ __device__ int x() const { return (D + kMxUnit - 1) / kMxUnit * kMxUnit * 2; }
    __host__ __device__ int bytes() const { return x() + kTBWarps * 512 + 8 * Kp * 4; }
};

// As k_token_block: a CTA walks one token down the tree and evaluates its leaf, with the arithmetic of k_leaf_mx4 on one token (its row
// is every column of the MMAs' operand; what the other seven columns give is not stored).  Three CTAs per SM (80 registers; 8 bytes
// spilled for leaves of up to 16, 24 of up to 32, 144 of wider ones): two are 2 us ahead up to two per SM and a fifth behind from then on, four behind
// everywhere.
template <int MT, bool kWide, bool kBig>
__global__ void __launch_bounds__(kTBThreads, 3)
k_mx4_token(const MxTokenArgs A)
{
    using T = __nv_bfloat16;
    constexpr bool K16 = MT == 1;
    constexpr int NW = kTBWarps, kSplit = NW / MT;
    extern __shared__ __align__(16) unsigned char smem_mt[];
    __shared__ float s_logit[2][8];
    __shared__ int s_tok[8];
    const MxLayout& Ly = A.lay;
    const int D = Ly.D, l = Ly.l, Kp = K16 ? 16 : kWide ? Ly.Kp() : 32;
    const MxTokenSmem S{D, Kp};
    T* xs = reinterpret_cast<T*>(smem_mt);
    float* red = reinterpret_cast<float*>(smem_mt + S.x());              // [warp][register][lane]
    T* hid = reinterpret_cast<T*>(smem_mt + S.x() + NW * 512);           // [2][8][Kp]
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    TokenWalk<T> walk;
    walk.send_first(A.node_w, A.node_b, D, A.depth, true, warp, lane);
    for (int i = A.x_cols + tid; i < S.x() / 2; i += kTBThreads) xs[i] = __float2bfloat16_rn(0.0f);
    if (tid < 8) s_tok[tid] = blockIdx.x;
    pdl_trigger();
    pdl_wait();
    const T* xt = A.x + (int64_t)blockIdx.x * A.x_cols;
    if (A.x_cols == D) {
        for (int i = tid; i < D / 8; i += kTBThreads) reinterpret_cast<uint4*>(xs)[i] = __ldg(reinterpret_cast<const uint4*>(xt) + i);
    } else {
        for (int i = tid; i < A.x_cols; i += kTBThreads) xs[i] = xt[i];
    }
    __syncthreads();
    const int64_t leaf = walk.leaf(A.node_w, A.node_b, xs, D, A.depth, true, warp, lane, s_logit);
    if (tid == 0) {
        A.leaf_out[blockIdx.x] = (int32_t)leaf;
        if (A.leaf_out2) A.leaf_out2[blockIdx.x] = (int32_t)leaf;
    }
    const unsigned char* rec = A.image + leaf * Ly.record();
    const int at_s1 = Ly.at_s1(), at_b1 = Ly.at_b1(), units1 = Ly.units1();
    MxNext next;
    for (int unit0 = 0; unit0 < l; unit0 += 16 * MT) {
        const int row0 = unit0 + 16 * (warp / kSplit), u0 = warp % kSplit;
        MxCodes q;
#pragma unroll
        for (int k = 0; k < kMxAhead; ++k) mx_fetch_codes(rec, at_s1, l, row0, u0 + k * kSplit, units1, lane, q, k);
        if (unit0 == 0) mx_fetch_outputs<K16>(Ly, rec, warp, 0, lane, next);
        float acc[2][4] = {};
        mx_hidden<kBig, 2>(rec, at_s1, l, q, reinterpret_cast<const unsigned char*>(xs), 0, 1, row0, u0, units1, kSplit, 0, lane, acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) red[(warp * 4 + i) * 32 + lane] = acc[0][i];
        __syncthreads();
        for (int f = warp; f < 4 * MT; f += NW) {          // unit group, register; the lane is the lane
            const int m = f >> 2, i = f & 3, unit = unit0 + 16 * m + g + 8 * (i >> 1), row = 2 * c + (i & 1);
            float sum = unit < l ? __bfloat162float(__ldg(reinterpret_cast<const T*>(rec + at_b1) + unit)) : 0.0f;
#pragma unroll
            for (int w = 0; w < kSplit; ++w) sum += red[((m * kSplit + w) * 4 + i) * 32 + lane];
            const float h = unit < l ? activate_bf16(A.act, sum) : 0.0f;
            const T hi = __float2bfloat16_rn(h);
            const float f32 = __bfloat162float(hi);
            hid[row * Kp + unit] = hi;
            hid[(8 + row) * Kp + unit] = __float2bfloat16_rn(isinf(f32) ? 0.0f : h - f32);
        }
        __syncthreads();
    }
    mx_outputs<K16, kWide, kBig, 1>(A.y, A.y_vec, Ly, rec, hid, 8, 1, s_tok, warp, NW, lane, next);
}

// ---- thin leaves on CUDA cores ---------------------------------------------------------------------

struct MxRowsArgs {
    const __nv_bfloat16* x;
    const int32_t *leaf_idx, *perm;    // perm nullptr: in order
    const unsigned char* image;
    __nv_bfloat16* y;
    MxLayout lay;
    int act;
    int64_t B;
    bool y_vec, big;                   // rows of y are 16-byte vectors
    // the last levels of the walk, where the descent left some: from position pos[t] (0 without) of level level0
    const __nv_bfloat16 *node_w, *node_b;
    int level0, levels;
    const int32_t* pos;
    int32_t* leaf_out;
};

constexpr int kMxRowWarps = 8;

// Eight weights of a word, scaled.
__device__ __forceinline__ void mx_floats(uint32_t w, uint32_t sc, bool big, float (&v)[8]) {
    uint32_t r[4];
    mx_expand(w, r);
    const uint32_t f1 = mx_mul1(sc, big);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint32_t q = mul_bf16x2(r[p], f1);
        if (big) q = mul_bf16x2(q, mx_mul2(sc));
        v[2 * p] = __uint_as_float(q << 16);
        v[2 * p + 1] = __uint_as_float(q & 0xffff0000u);
    }
}

// A warp per token, in float32: leaves of fewer than 8 neurons have nothing to fill an MMA with, and with about a token per leaf the
// work is a gather of weights.  Lanes take eight columns of x (then eight outputs) each, one word of codes per row.
// Dynamic shared memory: kMxRowWarps * l floats.  The walk is that of k_leaf_warp.
template <bool kTail>
__global__ void __launch_bounds__(kMxRowWarps * 32, 4)
k_leaf_mx4_rows(const MxRowsArgs A)
{
    extern __shared__ float s_mxh[];
    pdl_trigger();
    pdl_wait();
    constexpr int U = 2;                                   // rows of W1 that share the loads of x
    const MxLayout& Ly = A.lay;
    const int lane = threadIdx.x & 31, wib = threadIdx.x >> 5, D = Ly.D, O = Ly.O, l = Ly.l;
    const int wd = (D + 7) / 8, wo = (O + 7) / 8, nd = (int)mx_scales(D), no = (int)mx_scales(O);
    const int64_t record = Ly.record();
    float* h = s_mxh + (size_t)wib * l;
    for (int64_t i = (int64_t)blockIdx.x * kMxRowWarps + wib; i < A.B; i += (int64_t)gridDim.x * kMxRowWarps) {
        const int64_t t = A.perm ? A.perm[i] : i;
        const __nv_bfloat16* xt = A.x + t * D;
        int64_t j;
        if (kTail) {
            int64_t n = A.pos ? A.pos[t] : 0;
            for (int m = A.level0; m < A.level0 + A.levels; ++m) {
                const int64_t row = ((int64_t)1 << m) - 1 + n;
                const float logit = warp_dot<__nv_bfloat16>(A.node_w + row * D, xt, D, true, lane) + __bfloat162float(A.node_b[row]);
                n = 2 * n + (logit >= 0.0f ? 1 : 0);
            }
            j = n;
            if (lane == 0) A.leaf_out[t] = (int32_t)n;
        } else {
            j = A.leaf_idx[t];
        }
        const unsigned char* rec = A.image + j * record;
        if (lane == 0) mx_prefetch(rec, record);
        const uint32_t *w1 = reinterpret_cast<const uint32_t*>(rec), *w2 = reinterpret_cast<const uint32_t*>(rec + Ly.at_w2());
        const uint8_t *s1 = rec + Ly.at_s1(), *s2 = rec + Ly.at_s2();
        const __nv_bfloat16 *b1 = reinterpret_cast<const __nv_bfloat16*>(rec + Ly.at_b1()), *b2 = reinterpret_cast<const __nv_bfloat16*>(rec + Ly.at_b2());
        for (int i0 = 0; i0 < l; i0 += U) {
            float acc[U] = {};
            for (int w = lane; w < wd; w += 32) {
                float xv[8];
                Elem<__nv_bfloat16>::load_vec(xt + 8 * w, xv);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (i0 + u >= l) break;
                    float v[8];
                    mx_floats(__ldg(w1 + (int64_t)(i0 + u) * wd + w), __ldg(s1 + (i0 + u) * nd + (w >> 2)), A.big, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[u] = fmaf(v[e], xv[e], acc[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float sum = warp_sum(acc[u]);
                if (lane == 0 && i0 + u < l) h[i0 + u] = activate(A.act, sum + __bfloat162float(b1[i0 + u]));
            }
        }
        __syncwarp();
        __nv_bfloat16* yt = A.y + t * O;
        for (int w = lane; w < wo; w += 32) {
            float acc[8];
            Elem<__nv_bfloat16>::load_vec(b2 + 8 * w, acc);
            for (int q = 0; q < l; ++q) {
                float v[8];
                mx_floats(__ldg(w2 + (int64_t)q * wo + w), __ldg(s2 + q * no + (w >> 2)), A.big, v);
                const float hq = h[q];
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = fmaf(v[e], hq, acc[e]);
            }
            if (A.y_vec) {
                *reinterpret_cast<uint4*>(yt + 8 * w) = make_uint4(ptx::pack_bf16(acc[0], acc[1]), ptx::pack_bf16(acc[2], acc[3]),
                                                                   ptx::pack_bf16(acc[4], acc[5]), ptx::pack_bf16(acc[6], acc[7]));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (8 * w + e < O) yt[8 * w + e] = __float2bfloat16_rn(acc[e]);
            }
        }
        __syncwarp();
    }
}

// The same for a few tokens, as k_mx4_token: a CTA per token, a warp per hidden unit, a thread per eight outputs.
__global__ void __launch_bounds__(kTBThreads, 4)
k_mx4_token_rows(const MxTokenArgs A)
{
    using T = __nv_bfloat16;
    extern __shared__ __align__(16) unsigned char smem_mt[];
    __shared__ float s_logit[2][8], s_h[8];
    const MxLayout& Ly = A.lay;
    const int D = Ly.D, O = Ly.O, l = Ly.l, wd = (D + 7) / 8, wo = (O + 7) / 8;
    T* xs = reinterpret_cast<T*>(smem_mt);                 // [8 wd]
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    TokenWalk<T> walk;
    walk.send_first(A.node_w, A.node_b, D, A.depth, true, warp, lane);
    if (tid < D - A.x_cols) xs[A.x_cols + tid] = __float2bfloat16_rn(0.0f);
    pdl_trigger();
    pdl_wait();
    const T* xt = A.x + (int64_t)blockIdx.x * A.x_cols;
    if (A.x_cols == D) {
        for (int i = tid; i < D / 8; i += kTBThreads) reinterpret_cast<uint4*>(xs)[i] = __ldg(reinterpret_cast<const uint4*>(xt) + i);
    } else {
        for (int i = tid; i < A.x_cols; i += kTBThreads) xs[i] = xt[i];
    }
    __syncthreads();
    const int64_t leaf = walk.leaf(A.node_w, A.node_b, xs, D, A.depth, true, warp, lane, s_logit);
    if (tid == 0) {
        A.leaf_out[blockIdx.x] = (int32_t)leaf;
        if (A.leaf_out2) A.leaf_out2[blockIdx.x] = (int32_t)leaf;
    }
    const unsigned char* rec = A.image + leaf * Ly.record();
    if (tid == 0) mx_prefetch(rec, Ly.record());
    if (warp < l) {
        const uint32_t* w1 = reinterpret_cast<const uint32_t*>(rec) + warp * wd;
        const unsigned char* s1 = rec + Ly.at_s1() + warp * (int)mx_scales(D);
        float sum = 0.0f;
#pragma unroll 4
        for (int w = lane; w < wd; w += 32) {
            float v[8], xv[8];
            mx_floats(__ldg(w1 + w), __ldg(s1 + (w >> 2)), A.big, v);
            Elem<T>::unpack(*reinterpret_cast<const uint4*>(xs + 8 * w), xv);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(v[e], xv[e], sum);
        }
        sum = warp_sum(sum);
        if (lane == 0) s_h[warp] = activate(A.act, sum + __bfloat162float(reinterpret_cast<const T*>(rec + Ly.at_b1())[warp]));
    }
    __syncthreads();
    const uint32_t* w2 = reinterpret_cast<const uint32_t*>(rec + Ly.at_w2());
    const unsigned char* s2 = rec + Ly.at_s2();
    const int no = (int)mx_scales(O);
    T* yt = A.y + (int64_t)blockIdx.x * O;
    for (int w = tid; w < wo; w += kTBThreads) {
        float acc[8];
        Elem<T>::load_vec(reinterpret_cast<const T*>(rec + Ly.at_b2()) + 8 * w, acc);
#pragma unroll 4
        for (int q = 0; q < l; ++q) {
            float v[8];
            mx_floats(__ldg(w2 + q * wo + w), __ldg(s2 + q * no + (w >> 2)), A.big, v);
            const float hq = s_h[q];
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf(v[e], hq, acc[e]);
        }
        const uint32_t out[4] = {ptx::pack_bf16(acc[0], acc[1]), ptx::pack_bf16(acc[2], acc[3]), ptx::pack_bf16(acc[4], acc[5]),
                                 ptx::pack_bf16(acc[6], acc[7])};
        mx_store8(yt + 8 * w, O - 8 * w, A.y_vec, out);
    }
}

}  // namespace fff
