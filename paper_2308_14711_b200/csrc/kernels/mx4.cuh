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

// Eight elements per thread, four threads per block.  Whole: rows of whole blocks, i.e. one long run of 16-byte vectors;
// otherwise rows start anywhere and end inside a block.  Bound: HBM.
template <typename T, bool kWhole>
__global__ void __launch_bounds__(256)
k_quantize_mx4(const T* __restrict__ src, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, T* __restrict__ values, int64_t rows,
               int64_t cols)
{
    pdl_trigger();
    pdl_wait();
    const int64_t nb = mx_scales(cols), cb = mx_code_bytes(cols), total = rows * nb * 4;
    const int64_t step = (int64_t)gridDim.x * blockDim.x;
    constexpr int U = 2;                                   // groups whose loads are in flight
    // (whole warps: the shuffles below want all lanes; U * step is a multiple of 32, and so is the rounded total)
    const int64_t end = (total + 31) & ~(int64_t)31;
    for (int64_t u0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; u0 < end; u0 += U * step) {
        float v[U][8];
        int64_t at[U];
        int n[U];                                          // elements of the group that exist
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t unit = u0 + u * step;
            const int64_t row = kWhole ? 0 : unit / (nb * 4), c0 = kWhole ? unit * 8 : (unit - row * nb * 4) * 8;
            n[u] = unit < total ? (kWhole ? 8 : (int)max((int64_t)0, min((int64_t)8, cols - c0))) : 0;
            at[u] = kWhole ? c0 : row * cols + c0;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = 0.0f;
            if (kWhole) {
                if (n[u]) {
                    if constexpr (sizeof(T) == 2) {
                        Elem<T>::load_vec(src + at[u], v[u]);
                    } else {
                        const float4 a = __ldcs(reinterpret_cast<const float4*>(src + at[u])), b = __ldcs(reinterpret_cast<const float4*>(src + at[u]) + 1);
                        v[u][0] = a.x; v[u][1] = a.y; v[u][2] = a.z; v[u][3] = a.w; v[u][4] = b.x; v[u][5] = b.y; v[u][6] = b.z; v[u][7] = b.w;
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < n[u]) v[u][e] = load_float(src + at[u] + e);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t unit = u0 + u * step;
            unsigned a = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) a = max(a, __float_as_uint(v[u][e]) & 0x7fffffffu);
            if (unit - (threadIdx.x & 31) >= total) break;                    // (the same answer in a whole warp)
            a = max(a, __shfl_xor_sync(kFullMask, a, 1));
            a = max(a, __shfl_xor_sync(kFullMask, a, 2));
            const int s = mx_block_scale(a);
            const bool finite = s != 255;
            // 2^(127 - s): at most 2^127, and products of it are exact but for those far below the smallest code
            const float inv = finite ? __uint_as_float((unsigned)(254 - s) << 23) : 0.0f;
            uint32_t word = 0;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float2 q = finite ? make_float2(v[u][e] * inv, v[u][e + 1] * inv) : make_float2(0.0f, 0.0f);
                word |= (uint32_t)__nv_cvt_float2_to_fp4x2(q, __NV_E2M1, cudaRoundNearest) << (4 * e);
            }
            if (n[u] == 0) continue;
            const int64_t row = kWhole ? 0 : unit / (nb * 4), g = kWhole ? unit : unit - row * nb * 4;
            if constexpr (kWhole) {
                *reinterpret_cast<uint32_t*>(codes + unit * 4) = word;
            } else {
                uint8_t* to = codes + row * cb + g * 4;
                for (int e = 0; e < n[u]; e += 2) to[e >> 1] = (uint8_t)(word >> (4 * e));
            }
            if ((g & 3) == 0) scales[kWhole ? unit >> 2 : row * nb + (g >> 2)] = (uint8_t)s;
            if (values) {
                const float sc = mx_scale(s);
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = mx_code_value(word >> (4 * e)) * sc;
                if constexpr (kWhole && sizeof(T) == 2) {
                    uint4 q;
                    q.x = ptx::pack_bf16(o[0], o[1]); q.y = ptx::pack_bf16(o[2], o[3]); q.z = ptx::pack_bf16(o[4], o[5]); q.w = ptx::pack_bf16(o[6], o[7]);
                    __stcs(reinterpret_cast<uint4*>(values + at[u]), q);
                } else if constexpr (kWhole) {
                    __stcs(reinterpret_cast<float4*>(values + at[u]), make_float4(o[0], o[1], o[2], o[3]));
                    __stcs(reinterpret_cast<float4*>(values + at[u]) + 1, make_float4(o[4], o[5], o[6], o[7]));
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < n[u]) values[at[u] + e] = Elem<T>::from_float(o[e]);
                }
            }
        }
    }
}

template <typename T, bool kWhole>
__global__ void __launch_bounds__(256)
k_dequantize_mx4(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ values, int64_t rows, int64_t cols)
{
    pdl_trigger();
    pdl_wait();
    const int64_t nb = mx_scales(cols), cb = mx_code_bytes(cols), total = rows * nb * 4;
    for (int64_t unit = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; unit < total; unit += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = kWhole ? 0 : unit / (nb * 4), g = kWhole ? unit : unit - row * nb * 4;
        const int n = kWhole ? 8 : (int)max((int64_t)0, min((int64_t)8, cols - g * 8));
        if (n == 0) continue;
        uint32_t word = 0;
        if constexpr (kWhole) word = __ldcs(reinterpret_cast<const uint32_t*>(codes + unit * 4));
        else
            for (int e = 0; e < n; e += 2) word |= (uint32_t)codes[row * cb + g * 4 + (e >> 1)] << (4 * e);
        const float sc = mx_scale(__ldg(scales + (kWhole ? unit >> 2 : row * nb + (g >> 2))));
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = mx_code_value(word >> (4 * e)) * sc;
        T* to = values + (kWhole ? unit * 8 : row * cols + g * 8);
        if constexpr (kWhole && sizeof(T) == 2) {
            uint4 q;
            q.x = ptx::pack_bf16(o[0], o[1]); q.y = ptx::pack_bf16(o[2], o[3]); q.z = ptx::pack_bf16(o[4], o[5]); q.w = ptx::pack_bf16(o[6], o[7]);
            __stcs(reinterpret_cast<uint4*>(to), q);
        } else if constexpr (kWhole) {
            __stcs(reinterpret_cast<float4*>(to), make_float4(o[0], o[1], o[2], o[3]));
            __stcs(reinterpret_cast<float4*>(to) + 1, make_float4(o[4], o[5], o[6], o[7]));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) to[e] = Elem<T>::from_float(o[e]);
        }
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
// The same for two codes with scales of their own (low byte of lo and of hi).
__device__ __forceinline__ uint32_t mx_pair(uint32_t lo, uint32_t hi) { return (lo & 0xffffu) | (hi & 0xffff0000u); }

constexpr int kMxUnit = 64;            // columns of x per step of the first product, outputs per step of the second

// Sizes of the images of a layer.  Leaves of 8 neurons and more (tensor cores): the operands of mma.sync in the order in which a
// warp loads them.  Thinner ones (CUDA cores): rows.  In both a row's columns are padded with zero codes.
struct MxLayout {
    int D, O, l;
    bool mma;
    __host__ __device__ int units1() const { return (D + kMxUnit - 1) / kMxUnit; }
    __host__ __device__ int units2() const { return (O + kMxUnit - 1) / kMxUnit; }
    __host__ __device__ int Kp() const { return l <= 16 ? 16 : (l + 31) / 32 * 32; }      // hidden units as the second product sees them
    // per leaf, in bytes
    __host__ __device__ int64_t w1() const { return mma ? (int64_t)units1() * l * 32 : (int64_t)l * ((D + 7) / 8) * 4; }
    __host__ __device__ int64_t s1() const { return mma ? (int64_t)units1() * l * 2 : (int64_t)l * mx_scales(D); }
    __host__ __device__ int64_t w2() const { return mma ? (int64_t)units2() * Kp() * 32 : (int64_t)l * ((O + 7) / 8) * 4; }
    __host__ __device__ int64_t s2() const { return mma ? (int64_t)units2() * 2 * Kp() : (int64_t)l * mx_scales(O); }
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
                           const uint8_t* __restrict__ sc2, uint32_t* __restrict__ w1img, uint8_t* __restrict__ s1img,
                           uint32_t* __restrict__ w2img, uint8_t* __restrict__ s2img, MxLayout L, int64_t n_leaves, bool big)
{
    const int64_t i0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
    const int l = L.l, D = L.D, O = L.O;
    auto word_of = [&](const uint8_t* codes, int64_t row, int cols, int c0) {
        uint32_t c[8];
        for (int e = 0; e < 8; ++e) c[e] = caller_code(codes, row, cols, c0 + e);
        return mx_image_word(c);
    };
    if (!L.mma) {
        const int wd = (D + 7) / 8, wo = (O + 7) / 8;
        for (int64_t i = i0; i < n_leaves * l * wd; i += step) w1img[i] = word_of(w1, i / wd, D, (int)(i % wd) * 8);
        for (int64_t i = i0; i < n_leaves * l * wo; i += step) w2img[i] = word_of(w2, i / wo, O, (int)(i % wo) * 8);
        const int nd = (int)mx_scales(D), no = (int)mx_scales(O);
        for (int64_t i = i0; i < n_leaves * l * nd; i += step) s1img[i] = image_scale(sc1, i / nd, D, (int)(i % nd) * kMxBlock, big);
        for (int64_t i = i0; i < n_leaves * l * no; i += step) s2img[i] = image_scale(sc2, i / no, O, (int)(i % no) * kMxBlock, big);
        return;
    }
    // W1: [leaf][unit][row][quarter of the unit's 64 columns][2 words]
    const int64_t n1 = L.w1() / 4, n2 = L.w2() / 4;
    for (int64_t i = i0; i < n_leaves * n1; i += step) {
        const int64_t leaf = i / n1, k = i - leaf * n1;
        const int u = (int)(k / (l * 8)), row = (int)(k % (l * 8)) / 8, q = (int)(k & 7);
        w1img[i] = word_of(w1, leaf * l + row, D, u * kMxUnit + q * 8);
    }
    for (int64_t i = i0; i < n_leaves * L.s1(); i += step) {
        const int64_t leaf = i / L.s1(), k = i - leaf * L.s1();
        const int u = (int)(k / (l * 2)), row = (int)(k % (l * 2)) / 2, b = (int)(k & 1);
        s1img[i] = image_scale(sc1, leaf * l + row, D, u * kMxUnit + b * kMxBlock, big);
    }
    // W2: [leaf][unit of 64 outputs][block of 32 hidden units][half of the 8 output tiles][lane][4 words], a word: the 8 hidden units
    // 8c.. of one output; with 16 hidden units [leaf][unit][lane][4 words], a word: the 4 units 4c.. of two outputs.  Output of tile i
    // and lane (g, c): 16 (g / 2) + 2 i + g % 2.
    const int Kp = L.Kp();
    for (int64_t i = i0; i < n_leaves * n2; i += step) {
        const int64_t leaf = i / n2, k = i - leaf * n2;
        const int u = (int)(k / (Kp * 8)), in = (int)(k % (Kp * 8));
        const int j = in & 3, lane = (in >> 2) & 31, g = lane >> 2, c = lane & 3;
        uint32_t code[8];
        for (int e = 0; e < 8; ++e) {
            int tile, unit;
            if (Kp == 16) {
                tile = 2 * j + (e >> 2);
                unit = 4 * c + (e & 3);
            } else {
                const int kb = in >> 8, half = (in >> 7) & 1;
                tile = half * 4 + j;
                unit = kb * 32 + 8 * c + e;
            }
            const int o = u * kMxUnit + 16 * (g >> 1) + 2 * tile + (g & 1);
            code[e] = unit < l ? caller_code(w2, leaf * l + unit, O, o) : 0u;
        }
        w2img[i] = mx_image_word(code);
    }
    // [leaf][unit][half of its outputs][hidden unit]
    for (int64_t i = i0; i < n_leaves * L.s2(); i += step) {
        const int64_t leaf = i / L.s2(), k = i - leaf * L.s2();
        const int u = (int)(k / (2 * Kp)), b = (int)(k / Kp) & 1, unit = (int)(k % Kp);
        s2img[i] = unit < l ? image_scale(sc2, leaf * l + unit, O, u * kMxUnit + b * kMxBlock, big) : (uint8_t)(big ? 0 : 126);
    }
}

// ---- leaves on tensor cores ------------------------------------------------------------------------

struct MxLeafArgs {
    const __nv_bfloat16* x;
    const int32_t* perm;               // tokens in bucket order, or the table of lists [n_leaves][cap]
    const Tile* tiles;                 // (counts == nullptr) tile list
    int n_tiles;
    int32_t* counts;                   // entries of every list, [1] CTAs that have finished; zeroed at the end
    int n_leaves, cap;
    const uint32_t *w1, *w2;
    const uint8_t *s1, *s2;
    const __nv_bfloat16 *b1, *b2;      // caller layout
    __nv_bfloat16* y;
    MxLayout lay;
    int act, tile_rows;                // tile_rows: 32 or 64
    int x_bytes, y_bytes;              // widest access that rows of x / y allow: 32, 16 or 2
};

constexpr int kMxWarps = 8;
constexpr int kMxThreads = kMxWarps * 32;

// 16 consecutive columns of a row (columns past n read as zero).
__device__ __forceinline__ void mx_load16(const __nv_bfloat16* __restrict__ p, int n, int width, uint32_t (&r)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = 0u;
    if (width == 32) {
        if (n > 0)
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(p));
    } else if (width == 16) {
        if (n > 0) { const uint4 a = __ldg(reinterpret_cast<const uint4*>(p)); r[0] = a.x; r[1] = a.y; r[2] = a.z; r[3] = a.w; }
        if (n > 8) { const uint4 a = __ldg(reinterpret_cast<const uint4*>(p) + 1); r[4] = a.x; r[5] = a.y; r[6] = a.z; r[7] = a.w; }
    } else {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (2 * i < n) r[i] = __ldg(q + 2 * i);
            if (2 * i + 1 < n) r[i] |= (uint32_t)__ldg(q + 2 * i + 1) << 16;
        }
    }
}
__device__ __forceinline__ void mx_store16(__nv_bfloat16* __restrict__ p, int n, int width, const uint32_t (&r)[8]) {
    if (width == 32) {
        if (n > 0) ptx::st_global_v8(p, r);
    } else if (width == 16) {
        if (n > 0) __stcs(reinterpret_cast<uint4*>(p), make_uint4(r[0], r[1], r[2], r[3]));
        if (n > 8) __stcs(reinterpret_cast<uint4*>(p) + 1, make_uint4(r[4], r[5], r[6], r[7]));
    } else {
        uint16_t* q = reinterpret_cast<uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (2 * i < n) q[2 * i] = (uint16_t)r[i];
            if (2 * i + 1 < n) q[2 * i + 1] = (uint16_t)(r[i] >> 16);
        }
    }
}

// Shared memory of k_leaf_mx4: partial sums of the first product, hidden values (two bf16 planes), the tile's tokens, and the number
// of tiles before every leaf where tiles come from lists.
template <int NT>
struct MxLeafSmem {
    static constexpr int kRed = kMxWarps * 2 * NT * 4 * 32 * 4;
    __host__ __device__ static int hidden(int tile_rows, int Kp) { return tile_rows * Kp * 4; }
    __host__ __device__ static int bytes(int tile_rows, int Kp, int listed) {
        return kRed + hidden(tile_rows, Kp) + tile_rows * 4 + (listed ? (listed + 1) * 2 + 2 : 0);
    }
};

// Hidden layer of 32 rows and 8 NT units: this warp's share of the columns.  Token rows and codes go from global memory straight
// into the operands of the MMAs: the order of the summands is free, so lane c of a quad takes 16 consecutive columns of its row (32
// bytes of x, 8 of codes, one scale) for four MMAs.
template <int NT, bool kBig>
__device__ __forceinline__ void mx_hidden(const MxLeafArgs& A, const uint32_t* __restrict__ w1, const uint8_t* __restrict__ s1, const int (&tok)[4],
                                          int unit0, int warp, int lane, float (&acc)[2][NT][4])
{
    const int g = lane >> 2, c = lane & 3, l = A.lay.l, D = A.lay.D;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.0f;
    const bool two = __any_sync(kFullMask, tok[2] >= 0);
    for (int u = warp; u < A.lay.units1(); u += kMxWarps) {
        const int col = u * kMxUnit + 16 * c;
        uint32_t xr[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) mx_load16(A.x + (int64_t)max(tok[i], 0) * D + col, tok[i] >= 0 ? D - col : 0, A.x_bytes, xr[i]);
        uint2 code[NT];
        uint32_t sc[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int row = unit0 + 8 * j + g;
            const bool in = row < l;
            code[j] = in ? __ldg(reinterpret_cast<const uint2*>(w1) + ((int64_t)u * l + row) * 4 + c) : make_uint2(0u, 0u);
            sc[j] = in ? __ldg(s1 + ((int64_t)u * l + row) * 2 + (c >> 1)) : 0u;
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const uint32_t f1 = mx_mul1(sc[j], kBig), f2 = kBig ? mx_mul2(sc[j]) : 0u;
            uint32_t b[8];
            {
                uint32_t lo[4], hi[4];
                mx_expand(code[j].x, lo);
                mx_expand(code[j].y, hi);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    b[i] = mul_bf16x2(lo[i], f1);
                    b[4 + i] = mul_bf16x2(hi[i], f1);
                    if (kBig) { b[i] = mul_bf16x2(b[i], f2); b[4 + i] = mul_bf16x2(b[4 + i], f2); }
                }
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                ptx::mma_bf16(acc[0][j], xr[0][2 * s], xr[1][2 * s], xr[0][2 * s + 1], xr[1][2 * s + 1], b[2 * s], b[2 * s + 1]);
                if (two) ptx::mma_bf16(acc[1][j], xr[2][2 * s], xr[3][2 * s], xr[2][2 * s + 1], xr[3][2 * s + 1], b[2 * s], b[2 * s + 1]);
            }
        }
    }
}

// One K-block of the second product: the eight output tiles' operands from their words.  K16: 16 hidden units (two words' worth of
// tiles per word), else 32.
template <bool K16, bool kBig>
__device__ __forceinline__ void mx_output_operands(const uint4 (&word)[2], uint2 sc, uint32_t (&b)[8][K16 ? 2 : 4])
{
    // multipliers of the pairs of hidden units (the scales of a pair are neighbouring bytes)
    constexpr int P = K16 ? 2 : 4;
    uint32_t f1[P], f2[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const uint32_t two = p < 2 ? sc.x : sc.y, lo = (two >> (16 * (p & 1))) & 0xffu, hi = (two >> (16 * (p & 1) + 8)) & 0xffu;
        f1[p] = mx_pair(mx_mul1(lo, kBig), mx_mul1(hi, kBig));
        f2[p] = kBig ? mx_pair(mx_mul2(lo), mx_mul2(hi)) : 0u;
    }
    const uint32_t w[8] = {word[0].x, word[0].y, word[0].z, word[0].w, word[1].x, word[1].y, word[1].z, word[1].w};
#pragma unroll
    for (int i = 0; i < (K16 ? 4 : 8); ++i) {
        uint32_t r[4];
        mx_expand(w[i], r);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int tile = K16 ? 2 * i + (q >> 1) : i, p = K16 ? (q & 1) : q;
            uint32_t v = mul_bf16x2(r[q], f1[p]);
            if (kBig) v = mul_bf16x2(v, f2[p]);
            b[tile][p] = v;
        }
    }
}

// A CTA per tile of up to tile_rows tokens of one leaf.  The first product is split along D over the warps (no weight is expanded
// twice), their sums meet in shared memory, where bias and activation are applied; for the second product every warp has output
// columns of its own, numbered so that a lane ends with 16 consecutive outputs of its tokens.  Hidden values are kept as sums of two
// bf16 values (float32 precision to 2^-18): the extra MMAs cost little next to the expansion.
// NT: groups of 8 hidden units at a time: 2 for leaves of up to 16 (one K-block of 16 in the second product), else 4.
template <int NT, bool kBig>
__global__ void __launch_bounds__(kMxThreads, 2)
k_leaf_mx4(const MxLeafArgs A)
{
    using S = MxLeafSmem<NT>;
    constexpr bool K16 = NT == 2;
    extern __shared__ __align__(16) unsigned char smem_mx[];
    __shared__ int s_wsum[kMxWarps];
    const MxLayout& Ly = A.lay;
    const int Kp = Ly.Kp(), l = Ly.l, O = Ly.O;
    float* red = reinterpret_cast<float*>(smem_mx);                                   // [warp][m-tile, group, register][lane]
    __nv_bfloat16* hid = reinterpret_cast<__nv_bfloat16*>(smem_mx + S::kRed);         // [2][tile_rows][Kp]
    int* s_tok = reinterpret_cast<int*>(smem_mx + S::kRed + S::hidden(A.tile_rows, Kp));
    uint16_t* s_pre = reinterpret_cast<uint16_t*>(s_tok + A.tile_rows);
    const int plane = A.tile_rows * Kp;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    pdl_trigger();
    pdl_wait();
    if (A.counts) tiles_before_bins([&](int b) { return __ldcg(A.counts + b); }, A.n_leaves, A.tile_rows, s_pre, s_wsum, kMxThreads);
    const int n_tiles = A.counts ? s_pre[A.n_leaves] : A.n_tiles;
    const int units2 = Ly.units2(), kblocks = K16 ? 1 : Kp / 32;

    for (int tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
        int leaf, rows;
        const int32_t* list;
        if (A.counts) {
            leaf = bin_of_tile(s_pre, A.n_leaves, tile);
            const int first = (tile - s_pre[leaf]) * A.tile_rows;
            rows = min(A.tile_rows, __ldcg(A.counts + leaf) - first);
            list = A.perm + (int64_t)leaf * A.cap + first;
        } else {
            const Tile t = A.tiles[tile];
            leaf = t.bin;
            rows = t.rows;
            list = A.perm + t.start;
        }
        if (rows == 0) continue;                           // (a list of tiles may contain empty ones)
        if (tid < A.tile_rows) s_tok[tid] = tid < rows ? __ldcg(list + tid) : -1;
        const uint32_t* w1 = A.w1 + (int64_t)leaf * (Ly.w1() / 4);
        const uint32_t* w2 = A.w2 + (int64_t)leaf * (Ly.w2() / 4);
        const uint8_t* s1 = A.s1 + (int64_t)leaf * Ly.s1();
        const uint8_t* s2 = A.s2 + (int64_t)leaf * Ly.s2();
        // needed after the whole of the first product
        for (int64_t off = (int64_t)tid * 128; off < Ly.w2(); off += kMxThreads * 128)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const unsigned char*>(w2) + off));
        __syncthreads();

        // ---- hidden values
        for (int unit0 = 0; unit0 < l; unit0 += 8 * NT) {
            for (int m0 = 0; m0 < rows; m0 += 32) {
                int tok[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) tok[i] = m0 + 8 * i + g < A.tile_rows ? s_tok[m0 + 8 * i + g] : -1;
                float acc[2][NT][4];
                mx_hidden<NT, kBig>(A, w1, s1, tok, unit0, warp, lane, acc);
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) red[((warp * 2 + m) * NT * 4 + j * 4 + i) * 32 + lane] = acc[m][j][i];
                __syncthreads();
                with_activation(A.act, [&](auto act) {
#pragma unroll
                    for (int e = 0; e < NT; ++e) {
                        const int f = warp + kMxWarps * e;             // m-tile, group, register; the lane is the lane
                        const int m = f / (NT * 4), j = (f >> 2) % NT, i = f & 3;
                        float sum = 0.0f;
#pragma unroll
                        for (int w = 0; w < kMxWarps; ++w) sum += red[(w * 2 * NT * 4 + f) * 32 + lane];
                        const int unit = unit0 + 8 * j + 2 * c + (i & 1), row = m0 + 16 * m + g + 8 * (i >> 1);
                        float h = 0.0f;
                        if (unit < l) h = activate(decltype(act)::value, sum + __bfloat162float(A.b1[(int64_t)leaf * l + unit]));
                        const float hi = __bfloat162float(__float2bfloat16_rn(h));
                        hid[row * Kp + unit] = __float2bfloat16_rn(h);
                        hid[plane + row * Kp + unit] = __float2bfloat16_rn(isinf(hi) ? 0.0f : h - hi);
                    }
                });
                __syncthreads();
            }
        }

        // ---- outputs
        for (int u = warp; u < units2; u += kMxWarps) {
            const int o = u * kMxUnit + 16 * c, n = O - o;
            uint32_t bias[8];
            mx_load16(A.b2 + (int64_t)leaf * O + o, n, O % 8 == 0 ? 16 : 2, bias);
            uint32_t b[8][K16 ? 2 : 4];
            auto operands = [&](int kb) {
                uint4 word[2];
                uint2 sc = make_uint2(0u, 0u);
                const uint4* src = reinterpret_cast<const uint4*>(w2) + ((int64_t)u * kblocks + kb) * (K16 ? 32 : 64) + lane;
                word[0] = __ldg(src);
                word[1] = K16 ? make_uint4(0u, 0u, 0u, 0u) : __ldg(src + 32);
                const uint8_t* sp = s2 + ((int64_t)u * 2 + (g >> 2)) * Kp + kb * 32 + (K16 ? 4 : 8) * c;
                if (K16) sc.x = __ldg(reinterpret_cast<const uint32_t*>(sp));
                else sc = __ldg(reinterpret_cast<const uint2*>(sp));
                mx_output_operands<K16, kBig>(word, sc, b);
            };
            if (kblocks == 1) operands(0);
            for (int m0 = 0; m0 < rows; m0 += 16) {
                float acc[8][4];
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][k] = 0.0f;
                for (int kb = 0; kb < kblocks; ++kb) {
                    if (kblocks > 1) operands(kb);
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const __nv_bfloat16* h0 = hid + p * plane + (m0 + g) * Kp + kb * 32 + (K16 ? 4 : 8) * c;
                        if constexpr (K16) {
                            const uint2 a = *reinterpret_cast<const uint2*>(h0), d = *reinterpret_cast<const uint2*>(h0 + 8 * Kp);
#pragma unroll
                            for (int i = 0; i < 8; ++i) ptx::mma_bf16(acc[i], a.x, d.x, a.y, d.y, b[i][0], b[i][1]);
                        } else {
                            const uint4 a = *reinterpret_cast<const uint4*>(h0), d = *reinterpret_cast<const uint4*>(h0 + 8 * Kp);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                ptx::mma_bf16(acc[i], a.x, d.x, a.y, d.y, b[i][0], b[i][1]);
                                ptx::mma_bf16(acc[i], a.z, d.z, a.w, d.w, b[i][2], b[i][3]);
                            }
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int tok = s_tok[m0 + g + 8 * r];
                    uint32_t out[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        out[i] = ptx::pack_bf16(acc[i][2 * r] + __uint_as_float(bias[i] << 16), acc[i][2 * r + 1] + __uint_as_float(bias[i] & 0xffff0000u));
                    if (tok >= 0) mx_store16(A.y + (int64_t)tok * O + o, n, A.y_bytes, out);
                }
            }
        }
        __syncthreads();
    }
    // the last CTA to finish clears the counts (and the word behind them that counts the CTAs) for the next call
    if (A.counts) {
        __shared__ int s_last;
        __syncthreads();
        if (tid == 0) {
            __threadfence();
            s_last = atomicAdd(A.counts + A.n_leaves, 1) == (int)gridDim.x - 1 ? 1 : 0;
        }
        __syncthreads();
        if (s_last)
            for (int b = tid; b <= A.n_leaves; b += kMxThreads) A.counts[b] = 0;
    }
}

// ---- thin leaves on CUDA cores ---------------------------------------------------------------------

struct MxRowsArgs {
    const __nv_bfloat16* x;
    const int32_t *leaf_idx, *perm;    // perm nullptr: in order
    const uint32_t *w1, *w2;
    const uint8_t *s1, *s2;
    const __nv_bfloat16 *b1, *b2;
    __nv_bfloat16* y;
    MxLayout lay;
    int act;
    int64_t B;
    bool x_vec, y_vec, big;            // rows of x / y are 16-byte vectors
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
    float* h = s_mxh + (size_t)wib * l;
    auto load8 = [&](const __nv_bfloat16* p, int n, bool vec, float (&v)[8]) {
        if (vec) {
            Elem<__nv_bfloat16>::load_vec(p, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < n ? __bfloat162float(p[e]) : 0.0f;
        }
    };
    for (int64_t i = (int64_t)blockIdx.x * kMxRowWarps + wib; i < A.B; i += (int64_t)gridDim.x * kMxRowWarps) {
        const int64_t t = A.perm ? A.perm[i] : i;
        const __nv_bfloat16* xt = A.x + t * D;
        int64_t j;
        if (kTail) {
            int64_t n = A.pos ? A.pos[t] : 0;
            for (int m = A.level0; m < A.level0 + A.levels; ++m) {
                const int64_t row = ((int64_t)1 << m) - 1 + n;
                const float logit = warp_dot<__nv_bfloat16>(A.node_w + row * D, xt, D, A.x_vec, lane) + __bfloat162float(A.node_b[row]);
                n = 2 * n + (logit >= 0.0f ? 1 : 0);
            }
            j = n;
            if (lane == 0) A.leaf_out[t] = (int32_t)n;
        } else {
            j = A.leaf_idx[t];
        }
        const uint32_t *w1 = A.w1 + j * l * wd, *w2 = A.w2 + j * l * wo;
        const uint8_t *s1 = A.s1 + j * l * nd, *s2 = A.s2 + j * l * no;
        for (int i0 = 0; i0 < l; i0 += U) {
            float acc[U] = {};
            for (int w = lane; w < wd; w += 32) {
                float xv[8];
                load8(xt + 8 * w, D - 8 * w, A.x_vec, xv);
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
                if (lane == 0 && i0 + u < l) h[i0 + u] = activate(A.act, sum + __bfloat162float(A.b1[j * l + i0 + u]));
            }
        }
        __syncwarp();
        __nv_bfloat16* yt = A.y + t * O;
        for (int w = lane; w < wo; w += 32) {
            float acc[8];
            load8(A.b2 + j * O + 8 * w, O - 8 * w, A.y_vec, acc);
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

}  // namespace fff
