// The balance loss of a batch's routing, and the gradients of losses on the mixture weights.
//
// A token b has mixture weights mix[b, j] over the L = 2^d leaves (FORWARD_T) and the leaf that FORWARD_I gives it.  Over the n
// tokens that count (mask not zero, leaf in range):
//     counts_j = tokens of leaf j,   f_j = counts_j / n,   P_j = mean of mix[., j],   loss = L sum_j f_j P_j,
// smallest (1) where the leaves share tokens and weight evenly.  f is a count and carries no gradient:
//     d loss / d mix[b, j] = L f_j / n  for a token that counts, 0 otherwise.
// From the mixture weights back to the node logits: with g_j = d loss / d mix_j, and M and S the sums of mix_j and mix_j g_j over the
// leaves below a child, the node's choice is c = M_right / (M_left + M_right) and
//     d loss / d z = sum_j g_j d mix_j / d z = S_right (1 - c) - S_left c,
// which needs no logits: one pass over the mixture weights, bottom-up.
//
// All three are bound by HBM: 4 B L bytes are read (twice that with a second gradient) or written, a few operations each.
#pragma once

#include <float.h>

#include "common.cuh"

namespace fff {

// ---- balance loss ----------------------------------------------------------------------------------

constexpr int kBalThreads = 512;
constexpr int kBalCols = 512;                 // columns (leaves) per tile
constexpr int kBalGroup = 16;                 // slices that one CTA adds up
// Row slices per tile: two CTAs per SM.
__host__ inline int balance_max_slices(int tiles) { return tiles < 296 ? 296 / tiles : 1; }
__host__ __device__ inline int balance_groups(int slices) { return (slices + kBalGroup - 1) / kBalGroup; }

struct BalanceScratch {
    float2* parts;          // [slices][L] sum of mix_j, tokens of leaf j (as int bits)
    double* group_sums;     // [groups][L] the same of a group of slices
    int32_t* group_counts;  // [groups][L]
    int32_t* rows;          // [tiles][slices] tokens that count
    int32_t* group_rows;    // [tiles][groups]
    double* loss;           // [tiles] sum of counts_j * (sum of mix_j)
    int* done;              // [tiles][groups + 1] + [1], zero between calls
};

// What says whether a token counts.  (Loads without branches: a branch around one has the next one wait for it.)
struct TokenFlags {
    int leaf, kept;
    __device__ __forceinline__ bool counts(int n_leaves) const { return (unsigned)leaf < (unsigned)n_leaves && kept; }
};
__device__ __forceinline__ TokenFlags token_flags(const int32_t* __restrict__ leaf_idx, const uint8_t* __restrict__ mask, int64_t b) {
    return TokenFlags{leaf_idx ? __ldg(leaf_idx + b) : 0, mask ? __ldg(mask + b) : 1};
}

// Grid (slices, tiles).  Every CTA adds up its rows of its columns and counts its rows' leaves among them; the last CTA of a tile
// adds up the slices in their order, the last tile the tiles: one launch, and the same bits every time.
// V: columns per thread (4; 1 for one or two leaves).  Rows are added in float32 (at most a few hundred each), slices in float64.
template <int V>
__global__ void __launch_bounds__(kBalThreads, 2)
k_balance_loss(const float* __restrict__ mix, const int32_t* __restrict__ leaf_idx, const uint8_t* __restrict__ mask,
               float* __restrict__ loss, int32_t* __restrict__ counts, float* __restrict__ mean, int64_t B, int n_leaves,
               BalanceScratch ws)
{
    constexpr int U = 8;                                  // rows whose loads are in flight
    __shared__ int s_hist[kBalCols];
    __shared__ float s_sum[kBalThreads * V], s_part[kBalThreads];
    __shared__ double s_loss[kBalThreads / 32];
    __shared__ int s_rows, s_last;
    const int tid = threadIdx.x;
    const int cols = min(n_leaves, kBalCols), col0 = blockIdx.y * cols;
    const int across = cols / V, down = kBalThreads / across;            // threads per row, rows at a time (powers of two)
    const int c = tid & (across - 1), r = tid / across;
    const int slices = gridDim.x, tiles = gridDim.y;
    const int64_t per = (B + slices - 1) / slices, b0 = blockIdx.x * per, b1 = min(B, b0 + per);
    for (int i = tid; i < cols; i += kBalThreads) s_hist[i] = 0;
    if (tid == 0) s_rows = 0;
    __syncthreads();
    pdl_trigger();
    pdl_wait();

    float acc[V];
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0.0f;
    int mine = 0;
    const float* base = mix + col0 + c * V;
    for (int64_t b = b0 + r; b < b1; b += (int64_t)U * down) {
        float m[U][V];
        TokenFlags flags[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = min(b + (int64_t)u * down, b1 - 1);      // (past the end: the last row again)
            flags[u] = token_flags(leaf_idx, mask, row);
            if constexpr (V == 4) {
                const float4 q = __ldcs(reinterpret_cast<const float4*>(base + row * n_leaves));
                m[u][0] = q.x; m[u][1] = q.y; m[u][2] = q.z; m[u][3] = q.w;
            } else {
                m[u][0] = __ldcs(base + row * n_leaves);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = b + (int64_t)u * down < b1 && flags[u].counts(n_leaves);
            // (rows that do not count are left out, not multiplied by zero: they may hold anything)
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] += in ? m[u][v] : 0.0f;
            if (c == 0 && in) {
                ++mine;
                if ((unsigned)(flags[u].leaf - col0) < (unsigned)cols) atomicAdd(&s_hist[flags[u].leaf - col0], 1);
            }
        }
    }
    if (mine) atomicAdd(&s_rows, mine);
#pragma unroll
    for (int v = 0; v < V; ++v) s_sum[(r * across + c) * V + v] = acc[v];          // [down][cols]
    __syncthreads();
    // V rows per thread, the lanes of a warp that have the same column, then at most 32 partial sums per column
    const int i = tid & (cols - 1), r2 = tid / cols;
    const int parts = cols < 32 ? kBalThreads / 32 : kBalThreads / cols;
    {
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) sum += s_sum[(r2 * V + v) * cols + i];
        for (int o = cols; o < 32; o <<= 1) sum += __shfl_xor_sync(kFullMask, sum, o);
        if (cols >= 32 || (tid & 31) < cols) s_part[(cols < 32 ? tid >> 5 : r2) * cols + i] = sum;
    }
    __syncthreads();
    float mine_sum = 0.0f;
    if (tid < cols)
        for (int k = 0; k < parts; ++k) mine_sum += s_part[k * cols + i];
    double sum = (double)mine_sum;
    int cnt = tid < cols ? s_hist[i] : 0;
    // Slices are added up by the last CTA of their group, groups by the last of the tile (148 slices by one CTA alone: 8 us).
    const int groups = balance_groups(slices), group = blockIdx.x / kBalGroup, first = group * kBalGroup;
    const int members = min(kBalGroup, slices - first);
    int* done = ws.done + blockIdx.y * (groups + 1);
    // whether this CTA is the last of `of` to have written what it has, which it then sees
    auto last_of = [&](int* counter, int of) {
        __threadfence();
        __syncthreads();
        if (tid == 0) {
            s_last = atomicAdd(counter, 1) == of - 1;
            if (s_last) { *counter = 0; s_rows = 0; }
        }
        __syncthreads();
        if (s_last) __threadfence();
        return s_last;
    };
    __shared__ double s_col[kBalThreads];
    __shared__ int s_cnt[kBalThreads];
    const int each = kBalThreads / cols;                  // threads per column
    // what the threads of a column have, in the column's first
    auto add_columns = [&](int of) {
        s_col[tid] = sum;
        s_cnt[tid] = cnt;
        __syncthreads();
        if (tid < cols)
            for (int k = 1; k < min(each, of); ++k) {
                sum += s_col[k * cols + i];
                cnt += s_cnt[k * cols + i];
            }
    };
    if (slices > 1) {
        if (tid < cols) ws.parts[(int64_t)blockIdx.x * n_leaves + col0 + i] = make_float2(mine_sum, __int_as_float(cnt));
        if (tid == 0) ws.rows[blockIdx.y * slices + blockIdx.x] = s_rows;
        if (!last_of(done + group, members)) return;
        if (tid < members) atomicAdd(&s_rows, __ldcg(ws.rows + blockIdx.y * slices + first + tid));
        float2 part[kBalGroup];
#pragma unroll
        for (int k = 0; k < kBalGroup; ++k)
            part[k] = r2 + k * each < members ? __ldcg(ws.parts + (int64_t)(first + r2 + k * each) * n_leaves + col0 + i) : make_float2(0.0f, 0.0f);
        sum = 0.0;
        cnt = 0;
#pragma unroll
        for (int k = 0; k < kBalGroup; ++k) {
            sum += (double)part[k].x;
            cnt += __float_as_int(part[k].y);
        }
        add_columns(members);
        if (groups > 1) {
            if (tid < cols) {
                ws.group_sums[(int64_t)group * n_leaves + col0 + i] = sum;
                ws.group_counts[(int64_t)group * n_leaves + col0 + i] = cnt;
            }
            if (tid == 0) ws.group_rows[blockIdx.y * groups + group] = s_rows;
            if (!last_of(done + groups, groups)) return;
            if (tid < groups) atomicAdd(&s_rows, __ldcg(ws.group_rows + blockIdx.y * groups + tid));
            sum = 0.0;
            cnt = 0;
#pragma unroll 10
            for (int k = r2; k < groups; k += each) {
                sum += __ldcg(ws.group_sums + (int64_t)k * n_leaves + col0 + i);
                cnt += __ldcg(ws.group_counts + (int64_t)k * n_leaves + col0 + i);
            }
            add_columns(groups);
        }
    }
    __syncthreads();
    const double n = (double)s_rows, inv = n > 0.0 ? 1.0 / n : 0.0;
    double part = 0.0;
    if (tid < cols) {
        if (counts) counts[col0 + i] = cnt;
        if (mean) mean[col0 + i] = (float)(n > 0.0 ? sum * inv : 0.0);
        part = cnt == 0 ? 0.0 : (double)cnt * sum;        // (not 0 times a sum that overflowed)
    }
    int* all_done = ws.done + tiles * (groups + 1);
    // (the columns' warps, which come first)
    const int col_warps = (cols + 31) / 32;
    if ((tid >> 5) < col_warps) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) part += __shfl_down_sync(kFullMask, part, o);
        if ((tid & 31) == 0) s_loss[tid >> 5] = part;
    }
    __syncthreads();
    if (tid == 0) {
        double t = 0.0;
        for (int w = 0; w < col_warps; ++w) t += s_loss[w];
        if (tiles == 1) {
            if (loss) loss[0] = (float)((double)n_leaves * t * inv * inv);
        } else {
            ws.loss[blockIdx.y] = t;
            __threadfence();
            s_last = atomicAdd(all_done, 1) == tiles - 1;
        }
    }
    if (tiles == 1) return;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    double total = 0.0;
    for (int t = tid; t < tiles; t += kBalThreads) total += __ldcg(ws.loss + t);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_down_sync(kFullMask, total, o);
    if ((tid & 31) == 0) s_loss[tid >> 5] = total;
    __syncthreads();
    if (tid == 0) {
        double t = 0.0;
        for (int w = 0; w < min(kBalThreads / 32, (tiles + 31) / 32); ++w) t += s_loss[w];
        if (loss) loss[0] = (float)((double)n_leaves * t * inv * inv);
        *all_done = 0;
    }
}

// ---- its gradient ----------------------------------------------------------------------------------

constexpr int kSlopeThreads = 512;

// Tokens that count: the sum of the counts (all of which belong to such tokens).  By all threads of a CTA.
__device__ __forceinline__ double counted_tokens(const int32_t* __restrict__ counts, int n_leaves, long long* s_red) {
    const int tid = threadIdx.x;
    long long n = 0;
#pragma unroll 4
    for (int j = tid; j < n_leaves; j += blockDim.x) n += __ldg(counts + j);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(kFullMask, n, o);
    if ((tid & 31) == 0) s_red[tid >> 5] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < min((int)(blockDim.x >> 5), (n_leaves + 31) / 32); ++w) n += s_red[w];
    __syncthreads();
    return (double)n;
}

// Grid (slices, tiles) as above; every thread keeps the slope of its columns and writes it (or zero) into its rows.
template <int V>
__global__ void __launch_bounds__(kSlopeThreads, 4)
k_balance_loss_backward(const int32_t* __restrict__ leaf_idx, const uint8_t* __restrict__ mask, const int32_t* __restrict__ counts,
                        const float* __restrict__ dloss, float* __restrict__ dmix, int64_t B, int n_leaves)
{
    constexpr int U = 4;
    __shared__ long long s_red[kSlopeThreads / 32];
    const int tid = threadIdx.x;
    const int cols = min(n_leaves, kBalCols), col0 = blockIdx.y * cols;
    const int across = cols / V, down = kSlopeThreads / across;
    const int c = tid & (across - 1), r = tid / across;
    pdl_trigger();
    pdl_wait();
    const double n = counted_tokens(counts, n_leaves, s_red);
    const double scale = n > 0.0 ? (double)__ldg(dloss) * (double)n_leaves / (n * n) : 0.0;
    float slope[V];
#pragma unroll
    for (int v = 0; v < V; ++v) slope[v] = (float)(scale * (double)__ldg(counts + col0 + c * V + v));
    const int64_t per = (B + gridDim.x - 1) / gridDim.x, b0 = blockIdx.x * per, b1 = min(B, b0 + per);
    float* base = dmix + col0 + c * V;
    for (int64_t b = b0 + r; b < b1; b += (int64_t)U * down) {
        TokenFlags flags[U];
#pragma unroll
        for (int u = 0; u < U; ++u) flags[u] = token_flags(leaf_idx, mask, min(b + (int64_t)u * down, b1 - 1));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = b + (int64_t)u * down;
            if (row >= b1) break;
            const bool in = flags[u].counts(n_leaves);
            if constexpr (V == 4)
                __stcs(reinterpret_cast<float4*>(base + row * n_leaves),
                       in ? make_float4(slope[0], slope[1], slope[2], slope[3]) : make_float4(0.0f, 0.0f, 0.0f, 0.0f));
            else
                __stcs(base + row * n_leaves, in ? slope[0] : 0.0f);
        }
    }
}

// ---- back to the node logits -----------------------------------------------------------------------

// The balance loss's slope of every leaf, less their mean dloss / n: a slope that is the same for all leaves moves no logit, and
// without it the differences between leaves are exact, (L counts_j - n) dloss / n^2.  scale = dloss / n^2, 0 with n = 0.
__device__ __forceinline__ float centred_slope(int32_t count, int n_leaves, double n, double scale) {
    return (float)(scale * ((double)n_leaves * (double)count - n));
}
__device__ __forceinline__ double slope_scale(const float* __restrict__ dloss, double n) { return n > 0.0 ? (double)__ldg(dloss) / (n * n) : 0.0; }

__global__ void __launch_bounds__(1024)
k_balance_slope(const int32_t* __restrict__ counts, const float* __restrict__ dloss, float* __restrict__ slope, int n_leaves)
{
    __shared__ long long s_red[32];
    pdl_trigger();
    pdl_wait();
    const double n = counted_tokens(counts, n_leaves, s_red), g = slope_scale(dloss, n);
    for (int j = blockIdx.x * blockDim.x + threadIdx.x; j < n_leaves; j += gridDim.x * blockDim.x)
        slope[j] = centred_slope(__ldg(counts + j), n_leaves, n, g);
}

constexpr int kRouteThreads = 256;
constexpr int kRoutePerSm = 3;                // CTAs per SM
constexpr int kRouteWarps = kRouteThreads / 32;
constexpr int kRouteChunk = 512;              // leaves that one warp reduces at a time: four per lane and four times that, nine levels
constexpr int kRouteMaxStagedLeaves = 4096;   // trees whose rows of gradients go through shared memory

// Where rows of mixture weights are at most a chunk, a warp takes rows for itself; longer ones a CTA.  Rows that one of them takes at a
// time: where they are staged a multiple of four, so that their outputs start on a 16-byte boundary.
__host__ __device__ inline bool route_staged(int n_leaves) { return n_leaves <= kRouteMaxStagedLeaves; }
__host__ __device__ inline bool route_by_warps(int n_leaves) { return n_leaves <= kRouteChunk; }
__host__ __device__ inline int route_rows(int n_leaves) {
    if (route_by_warps(n_leaves)) return n_leaves >= kRouteChunk / 4 ? 4 : kRouteChunk / n_leaves;
    return !route_staged(n_leaves) ? 1 : n_leaves >= 2048 ? 4 : 8;
}
// Floats of shared memory: gradients (of every warp's rows, or of the CTA's), sums of the chunks, slopes.
struct RouteSmem {
    int n_leaves;
    bool balance;
    __host__ __device__ int out() const { return route_staged(n_leaves) ? (route_rows(n_leaves) * (n_leaves - 1) + 3) & ~3 : 0; }
    __host__ __device__ int outs() const { return route_by_warps(n_leaves) ? kRouteWarps * out() : out(); }
    __host__ __device__ int tops() const { return route_by_warps(n_leaves) ? 0 : 2 * route_rows(n_leaves) * (n_leaves / kRouteChunk); }
    __host__ __device__ int slopes() const { return balance && route_staged(n_leaves) ? n_leaves : 0; }
    __host__ __device__ size_t bytes() const { return sizeof(float) * (size_t)(outs() + ((tops() + 3) & ~3) + slopes()) + 16; }
};

// One node: sums over its two children's leaves in, its own out.  Children too small for float32 have no say.
__device__ __forceinline__ float node_gradient(float ml, float sl, float mr, float sr, float& m, float& s) {
    m = ml + mr;
    s = sl + sr;
    const float inv = rcp_approx(m);
    const float g = sr * (ml * inv) - sl * (mr * inv);
    return m < FLT_MIN ? 0.0f : g;
}

// Up to 512 mixture weights (whole rows, or a part of one), `base` on from the first row of a group of rows that ends at `elems`: the
// gradients of all their nodes to out (rows dense); mm, ss: the sums over a part of a row.  By one warp: every lane has four neighbouring
// leaves of each of four chunks of 128, two levels in its registers; then up to five across the lanes, the chunks shared out on the way:
// after the first step a lane goes on with two of the four, after the second with one, so that a level costs what its nodes do (every
// lane going on with all four: 20 nodes and 40 shuffles instead of 6 and 12); then up to two across the chunks.
template <bool kUp, bool kBal>
__device__ __forceinline__ void route_chunk(const float* __restrict__ gm, const float* __restrict__ gd, const int32_t* __restrict__ leaf_idx,
                                            const uint8_t* __restrict__ mask, const float* slopes, int64_t row0, int base, int elems, int depth,
                                            float* out, int lane, float& mm, float& ss)
{
    constexpr int U = 4;
    const int L = 1 << depth, N = L - 1;
    float m4[U][4], g4[U][4];
    int leaf[U], kept[U];                                  // of the lane's row (depth >= 2)
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int e = base + i * 128 + lane * 4;
#pragma unroll
        for (int k = 0; k < 4; ++k) { m4[i][k] = 0.0f; g4[i][k] = 0.0f; }
        leaf[i] = 0;
        kept[i] = 1;
        if (e >= elems) continue;
        if (kBal && leaf_idx) leaf[i] = __ldg(leaf_idx + row0 + (e >> depth));
        if (mask) kept[i] = __ldg(mask + row0 + (e >> depth));
        // (L = 2: a lane's four weights are two rows, and the last lane may have one)
        if (depth >= 2 || e + 4 <= elems) {
            const float4 q = __ldcs(reinterpret_cast<const float4*>(gm + e));
            m4[i][0] = q.x; m4[i][1] = q.y; m4[i][2] = q.z; m4[i][3] = q.w;
            if constexpr (kUp) {
                const float4 d = __ldcs(reinterpret_cast<const float4*>(gd + e));
                g4[i][0] = d.x; g4[i][1] = d.y; g4[i][2] = d.z; g4[i][3] = d.w;
            }
        } else {
            for (int k = 0; k < 2; ++k) {
                m4[i][k] = gm[e + k];
                if constexpr (kUp) g4[i][k] = gd[e + k];
            }
        }
    }
    if (kBal || mask) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int e = base + i * 128 + lane * 4;
            if (e >= elems) continue;
            if (depth >= 2) {
                if (kBal && (unsigned)leaf[i] < (unsigned)L) {
                    const float4 q = *reinterpret_cast<const float4*>(slopes + (e & (L - 1)));
                    g4[i][0] += q.x; g4[i][1] += q.y; g4[i][2] += q.z; g4[i][3] += q.w;
                }
                if (!kept[i]) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) m4[i][k] = g4[i][k] = 0.0f;
                }
                continue;
            }
#pragma unroll
            for (int k = 0; k < 4; k += 2) {               // (L = 2: two rows)
                if (e + k >= elems) break;
                const int64_t b = row0 + ((e + k) >> 1);
                if (kBal && (!leaf_idx || (unsigned)__ldg(leaf_idx + b) < 2u)) {
                    g4[i][k] += slopes[0];
                    g4[i][k + 1] += slopes[1];
                }
                if (mask && __ldg(mask + b) == 0) m4[i][k] = m4[i][k + 1] = g4[i][k] = g4[i][k + 1] = 0.0f;
            }
        }
    }
    float m[U], t[U];                                      // sums over the lane's four leaves
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int e = base + i * 128 + lane * 4, row = e >> depth, j = e & (L - 1);
        float ma, sa, mb, sb;
        const float (&w)[4] = m4[i];
        const float g0 = node_gradient(w[0], w[0] * g4[i][0], w[1], w[1] * g4[i][1], ma, sa);
        const float g1 = node_gradient(w[2], w[2] * g4[i][2], w[3], w[3] * g4[i][3], mb, sb);
        const float g2 = node_gradient(ma, sa, mb, sb, m[i], t[i]);
        if (e >= elems) continue;
        if (depth == 1) {
            out[row] = g0;
            if (e + 2 < elems) out[row + 1] = g1;
        } else {
            float* o = out + row * N;
            const int last = (1 << (depth - 1)) - 1 + (j >> 1);          // first of two nodes above the leaves
            o[last] = g0;
            o[last + 1] = g1;
            o[(1 << (depth - 2)) - 1 + (j >> 2)] = g2;
        }
    }
    // the node 2^(2 + k) leaves wide that leaf `at` of the chunk belongs to
    auto store = [&](int at, int k, float g) {
        const int e = base + at;
        if (e < elems) out[(e >> depth) * N + (1 << (depth - 2 - k)) - 1 + ((e & (L - 1)) >> (2 + k))] = g;
    };
    const bool r0 = lane & 1, r1 = lane & 2;
    mm = ss = 0.0f;
    if (depth < 3) return;
    float m2[2], t2[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        // chunk i stays with even lanes, chunk 2 + i with odd ones
        const float mo = __shfl_xor_sync(kFullMask, r0 ? m[i] : m[2 + i], 1), to = __shfl_xor_sync(kFullMask, r0 ? t[i] : t[2 + i], 1);
        const float mk = r0 ? m[2 + i] : m[i], tk = r0 ? t[2 + i] : t[i];
        const float g = node_gradient(r0 ? mo : mk, r0 ? to : tk, r0 ? mk : mo, r0 ? tk : to, m2[i], t2[i]);
        store((r0 ? 2 + i : i) * 128 + (lane & ~1) * 4, 1, g);
    }
    if (depth < 4) return;
    const int mine = ((r0 ? 2 : 0) + (r1 ? 1 : 0)) * 128;  // first leaf of the chunk that the lane goes on with
    auto up = [&](int lanes, bool right) {                 // one more level: with the lane that has the other child
        const float mo = __shfl_xor_sync(kFullMask, mm, lanes), so = __shfl_xor_sync(kFullMask, ss, lanes);
        return node_gradient(right ? mo : mm, right ? so : ss, right ? mm : mo, right ? ss : so, mm, ss);
    };
    {
        const float mo = __shfl_xor_sync(kFullMask, r1 ? m2[0] : m2[1], 2), to = __shfl_xor_sync(kFullMask, r1 ? t2[0] : t2[1], 2);
        const float mk = r1 ? m2[1] : m2[0], tk = r1 ? t2[1] : t2[0];
        const float g = node_gradient(r1 ? mo : mk, r1 ? to : tk, r1 ? mk : mo, r1 ? tk : to, mm, ss);
        store(mine + (lane & ~3) * 4, 2, g);
    }
#pragma unroll
    for (int k = 3; k <= 5; ++k) {
        if (k > depth - 2) return;
        const float g = up(1 << (k - 1), (lane >> (k - 1)) & 1);
        if (((lane >> 2) & ((1 << (k - 2)) - 1)) == 0) store(mine + (lane & ~((1 << k) - 1)) * 4, k, g);
    }
    // chunks 0 and 1, 2 and 3; then both pairs
    if (depth < 8) return;
    float g = up(2, r1);
    if ((lane & ~1) == 0) store(mine, 6, g);
    if (depth < 9) return;
    g = up(1, r0);
    if (lane == 0) store(mine, 7, g);
}

// n floats from shared to global memory (both on 16-byte boundaries), by `threads` threads.
__device__ __forceinline__ void route_copy(float* __restrict__ dst, const float* src, int n, int id, int threads) {
    for (int i = id; i < n >> 2; i += threads) __stcs(reinterpret_cast<float4*>(dst) + i, reinterpret_cast<const float4*>(src)[i]);
    for (int i = (n & ~3) + id; i < n; i += threads) dst[i] = src[i];
}

// kUp: dmixture given; kBal: counts and dloss given (slope_table for more than kRouteMaxStagedLeaves leaves).
// Rows of gradients are collected in shared memory and leave as aligned 16-byte vectors (a row has 2^d - 1 of them, so rows start
// anywhere).  Rows with a zero mask give zeros.
template <bool kUp, bool kBal>
__global__ void __launch_bounds__(kRouteThreads, kRoutePerSm)
k_routing_backward(const float* __restrict__ mix, const float* __restrict__ dmix, const int32_t* __restrict__ leaf_idx,
                   const uint8_t* __restrict__ mask, const int32_t* __restrict__ counts, const float* __restrict__ dloss,
                   const float* __restrict__ slope_table, float* __restrict__ dz, int64_t B, int depth)
{
    extern __shared__ __align__(16) float s_route[];
    __shared__ long long s_red[kRouteWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int L = 1 << depth, N = L - 1, R = route_rows(L);
    const bool staged = route_staged(L), by_warps = route_by_warps(L);
    const RouteSmem S{L, kBal};
    float* s_out = s_route + (by_warps ? warp * S.out() : 0);            // [R][N]
    float* s_top = s_route + S.outs();                                   // [2][R][chunks of a row]
    float* s_slope = s_top + ((S.tops() + 3) & ~3);                      // [L]
    const float* slopes = staged ? s_slope : slope_table;
    pdl_trigger();
    pdl_wait();
    if (kBal && staged) {
        const double n = counted_tokens(counts, L, s_red), g = slope_scale(dloss, n);
        for (int j = tid; j < L; j += kRouteThreads) s_slope[j] = centred_slope(__ldg(counts + j), L, n, g);
        __syncthreads();
    }
    const int64_t groups = (B + R - 1) / R;
    float mm, ss;
    if (by_warps) {
        for (int64_t grp = (int64_t)blockIdx.x + (int64_t)gridDim.x * warp; grp < groups; grp += (int64_t)gridDim.x * kRouteWarps) {
            const int64_t row0 = grp * R;
            const int rows = (int)min((int64_t)R, B - row0), elems = rows * L;
            for (int base = 0; base < elems; base += kRouteChunk)
                route_chunk<kUp, kBal>(mix + row0 * L, kUp ? dmix + row0 * L : nullptr, leaf_idx, mask, slopes, row0, base, elems, depth, s_out, lane, mm, ss);
            __syncwarp();
            route_copy(dz + row0 * N, s_out, rows * N, lane, 32);
            __syncwarp();
        }
        return;
    }
    const int chunks = L / kRouteChunk;
    for (int64_t grp = blockIdx.x; grp < groups; grp += gridDim.x) {
        const int64_t row0 = grp * R;
        const int rows = (int)min((int64_t)R, B - row0), elems = rows * L;
        float* out = staged ? s_out : dz + row0 * N;
        for (int u = warp; u < rows * chunks; u += kRouteWarps) {
            route_chunk<kUp, kBal>(mix + row0 * L, kUp ? dmix + row0 * L : nullptr, leaf_idx, mask, slopes, row0, u * kRouteChunk, elems, depth, out, lane, mm, ss);
            if (lane == 0) {
                s_top[u] = mm;                                           // u = row * chunks + chunk
                s_top[R * chunks + u] = ss;
            }
        }
        // the levels above the chunks: a warp per row, in place (a step's reads lie ahead of its writes)
        __syncthreads();
        for (int row = warp; row < rows; row += kRouteWarps) {
            float* tm = s_top + row * chunks;
            float* ts = tm + R * chunks;
            float* o = out + (int64_t)row * N;
            for (int nodes = chunks >> 1; nodes >= 1; nodes >>= 1) {
                for (int p0 = 0; p0 < nodes; p0 += 32) {
                    const int p = p0 + lane;
                    if (p < nodes) o[nodes - 1 + p] = node_gradient(tm[2 * p], ts[2 * p], tm[2 * p + 1], ts[2 * p + 1], mm, ss);
                    __syncwarp();
                    if (p < nodes) { tm[p] = mm; ts[p] = ss; }
                    __syncwarp();
                }
            }
        }
        __syncthreads();
        if (staged) {
            route_copy(dz + row0 * N, s_out, rows * N, tid, kRouteThreads);
            __syncthreads();
        }
    }
}

}  // namespace fff
