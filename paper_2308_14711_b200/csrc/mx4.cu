// Launchers of the microscaled 4-bit kernels (kernels/mx4.cuh); arguments are checked by their callers in fff_api.cu.
#include "kernels/mx4.cuh"

#include <algorithm>
#include <mutex>

#include "launch.h"

namespace fff {

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_mu;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Whether rows of `cols` bf16 values are 16-byte vectors.
bool whole_vectors(const void* p, int cols) { return cols % 8 == 0 && aligned(p, 16); }

constexpr int kMxSmemMost = 226 * 1024;                       // shared memory of a CTA that has an SM to itself, or shares it with another
constexpr int kMxTokenSmemMost = 100 * 1024;
constexpr int kMxSmemPair = (227 * 1024) / 2 - 1024 - 128;

MxLayout layout(const Mx4Layer& m) { return MxLayout{m.D, m.O, m.l, m.mma}; }

// CTAs for `units` threads' work, at most `per_sm` per SM.
unsigned spread(int64_t units, int threads, int sm_count, int per_sm) {
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>((units + threads - 1) / threads, (int64_t)sm_count * per_sm));
}

template <typename T>
cudaError_t quantize(const LaunchOn& on, const T* src, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales, T* values) {
    const unsigned grid = spread((rows * mx_scales(cols) * 4 + kMxAtOnce - 1) / kMxAtOnce, 256, on.sm_count, 8);
    const auto kern = cols % kMxBlock == 0 ? k_quantize_mx4<T, kMxWhole> : cols % 8 == 0 ? k_quantize_mx4<T, kMxGroups> : k_quantize_mx4<T, kMxAny>;
    return launch_on(on, kern, grid, 1, 256, 0, src, codes, scales, values, rows, cols);
}

template <typename T>
cudaError_t dequantize(const LaunchOn& on, const uint8_t* codes, const uint8_t* scales, T* values, int64_t rows, int64_t cols) {
    const unsigned grid = spread(rows * mx_scales(cols) * 4, 256, on.sm_count, 16);
    const auto kern =
        cols % kMxBlock == 0 ? k_dequantize_mx4<T, kMxWhole> : cols % 8 == 0 ? k_dequantize_mx4<T, kMxGroups> : k_dequantize_mx4<T, kMxAny>;
    return launch_on(on, kern, grid, 1, 256, 0, codes, scales, values, rows, cols);
}

template <int MT, bool kWide, bool kBig>
cudaError_t launch_tiles(const LaunchOn& on, const MxLeafArgs& a, int n_tiles) {
    const int smem = MxLeafSmem{a.tile_rows, a.lay.D, a.lay.Kp(), a.counts ? a.n_leaves : 0}.bytes();
    static bool raised[kMaxDevices] = {};
    {
        std::lock_guard<std::mutex> lk(g_mu);
        if (!raised[on.device]) {
            const cudaError_t e = cudaFuncSetAttribute(k_leaf_mx4<MT, kWide, kBig>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMxSmemMost);
            if (e != cudaSuccess) return e;
            raised[on.device] = true;
        }
    }
    const int per_sm = smem <= kMxSmemPair ? 2 : 1;
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>((int64_t)on.sm_count * per_sm, n_tiles));
    return launch_on(on, k_leaf_mx4<MT, kWide, kBig>, grid, 1, kMxThreads, (size_t)smem, a);
}

}  // namespace

cudaError_t quantize_mx4(const LaunchOn& on, const void* src, int elem_bytes, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales,
                         void* values) {
    return elem_bytes == 4 ? quantize(on, (const float*)src, rows, cols, codes, scales, (float*)values)
                           : quantize(on, (const __nv_bfloat16*)src, rows, cols, codes, scales, (__nv_bfloat16*)values);
}

cudaError_t dequantize_mx4(const LaunchOn& on, const uint8_t* codes, const uint8_t* scales, int elem_bytes, int64_t rows, int64_t cols,
                           void* values) {
    return elem_bytes == 4 ? dequantize(on, codes, scales, (float*)values, rows, cols)
                           : dequantize(on, codes, scales, (__nv_bfloat16*)values, rows, cols);
}

// (leaves of fewer than 8 neurons would leave most of an MMA's columns empty)
bool mx4_on_tensor_cores(int leaf_width) { return leaf_width >= 8; }

size_t mx4_image_bytes(const Mx4Layer& m, int64_t n_leaves) { return (size_t)layout(m).record() * (size_t)n_leaves; }
bool mx4_record_fits(const Mx4Layer& m) {
    return ((int64_t)m.l * ((int64_t)m.D + m.O) + 64 * (int64_t)m.l) * 4 < ((int64_t)1 << 30);
}

cudaError_t mx4_find_big(const uint8_t* scales, int64_t n, int* flag, int sm_count) {
    k_mx_find_big<<<spread(n, 256, sm_count, 8), 256>>>(scales, n, flag);
    return cudaGetLastError();
}

cudaError_t mx4_pack(const Mx4Layer& m, const uint8_t* w1, const uint8_t* s1, const uint8_t* w2, const uint8_t* s2, const void* b1,
                     const void* b2, int64_t n_leaves, int sm_count) {
    k_pack_mx4<<<(unsigned)sm_count * 8, 256>>>(w1, s1, w2, s2, (const uint16_t*)b1, (const uint16_t*)b2, m.image, layout(m), n_leaves, m.big);
    return cudaGetLastError();
}

// Most tokens (a multiple of 8) that a tile can have while two CTAs fit an SM; 32 at least.
int mx4_most_rows(const Mx4Layer& m, int n_leaves) {
    for (int rows = 8 * kMxMaxGroups; rows > 32; rows -= 8)
        if (MxLeafSmem{rows, m.D, layout(m).Kp(), n_leaves}.bytes() <= kMxSmemPair) return rows;
    return 32;
}

cudaError_t mx4_copy_rows(const LaunchOn& on, void* dst, int dst_cols, const void* src, int src_cols, int64_t rows) {
    return launch_on(on, k_mx4_copy_rows, spread(rows * (dst_cols <= 64 ? 8 : 32), 256, on.sm_count, 8), 1, 256, 0, (uint16_t*)dst, dst_cols, (const uint16_t*)src, src_cols,
                     rows);
}

cudaError_t mx4_leaf_tiles(const LaunchOn& on, const Mx4Layer& m, const Mx4Tokens& t, const int32_t* perm, const void* tiles, int n_tiles,
                           int tile_rows, int32_t* counts, int n_leaves, int cap) {
    MxLeafArgs a = {};
    a.x = (const __nv_bfloat16*)t.x;
    a.perm = perm;
    a.tiles = (const Tile*)tiles;
    a.n_tiles = n_tiles;
    a.counts = counts;
    a.n_leaves = n_leaves;
    a.cap = cap;
    a.image = m.image;
    a.y = (__nv_bfloat16*)t.y;
    a.lay = layout(m);
    a.act = t.act;
    a.tile_rows = tile_rows;
    a.y_vec = whole_vectors(t.y, m.O);
    a.status = t.status;
    if (m.l <= 16) return m.big ? launch_tiles<1, false, true>(on, a, n_tiles) : launch_tiles<1, false, false>(on, a, n_tiles);
    if (m.l <= 32) return m.big ? launch_tiles<2, false, true>(on, a, n_tiles) : launch_tiles<2, false, false>(on, a, n_tiles);
    return m.big ? launch_tiles<2, true, true>(on, a, n_tiles) : launch_tiles<2, true, false>(on, a, n_tiles);
}

namespace {

cudaError_t launch_token(const LaunchOn& on, void (*kern)(MxTokenArgs), int smem, const MxTokenArgs& a, int64_t B) {
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMxTokenSmemMost);
        if (e != cudaSuccess) return e;
    }
    return launch_on(on, kern, (unsigned)B, 1, kTBThreads, (size_t)smem, a);
}

template <int MT, bool kWide, bool kBig>
cudaError_t launch_token(const LaunchOn& on, const MxTokenArgs& a, int64_t B) {
    return launch_token(on, k_mx4_token<MT, kWide, kBig>, MxTokenSmem{a.lay.D, a.lay.Kp()}.bytes(), a, B);
}

}  // namespace

bool mx4_token_fits(const Mx4Layer& m) { return MxTokenSmem{m.D, layout(m).Kp()}.bytes() <= kMxTokenSmemMost; }

cudaError_t mx4_tokens(const LaunchOn& on, const Mx4Layer& m, const Mx4Tokens& t, const void* node_w, const void* node_b, int depth, int32_t* leaf_out,
                       int32_t* leaf_out2, int64_t B) {
    MxTokenArgs a = {};
    a.x = (const __nv_bfloat16*)t.x;
    a.node_w = (const __nv_bfloat16*)node_w;
    a.node_b = (const __nv_bfloat16*)node_b;
    a.image = m.image;
    a.y = (__nv_bfloat16*)t.y;
    a.leaf_out = leaf_out;
    a.leaf_out2 = leaf_out2;
    a.lay = layout(m);
    a.depth = depth;
    a.act = t.act;
    a.x_cols = t.x_cols;
    a.y_vec = whole_vectors(t.y, m.O);
    a.big = m.big;
    if (!m.mma) return launch_token(on, k_mx4_token_rows, MxTokenSmem{m.D, 0}.x(), a, B);
    if (m.l <= 16) return m.big ? launch_token<1, false, true>(on, a, B) : launch_token<1, false, false>(on, a, B);
    if (m.l <= 32) return m.big ? launch_token<2, false, true>(on, a, B) : launch_token<2, false, false>(on, a, B);
    return m.big ? launch_token<2, true, true>(on, a, B) : launch_token<2, true, false>(on, a, B);
}

cudaError_t mx4_leaf_rows(const LaunchOn& on, const Mx4Layer& m, const Mx4Tokens& t, const int32_t* leaf_idx, const int32_t* perm, int64_t B,
                          const Mx4Tail& tail) {
    MxRowsArgs a = {};
    a.x = (const __nv_bfloat16*)t.x;
    a.leaf_idx = leaf_idx;
    a.perm = perm;
    a.image = m.image;
    a.y = (__nv_bfloat16*)t.y;
    a.lay = layout(m);
    a.act = t.act;
    a.B = B;
    a.y_vec = whole_vectors(t.y, m.O);
    a.big = m.big;
    a.node_w = (const __nv_bfloat16*)tail.node_w;
    a.node_b = (const __nv_bfloat16*)tail.node_b;
    a.level0 = tail.level0;
    a.levels = tail.levels;
    a.pos = tail.pos;
    a.leaf_out = tail.leaf_out;
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>((B + kMxRowWarps - 1) / kMxRowWarps, (int64_t)on.sm_count * 8));
    return launch_on(on, tail.levels > 0 ? k_leaf_mx4_rows<true> : k_leaf_mx4_rows<false>, grid, 1, kMxRowWarps * 32,
                     sizeof(float) * (size_t)kMxRowWarps * m.l, a);
}

}  // namespace fff

