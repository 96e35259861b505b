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
// All three are bound by HBM: 4 B L bytes are read (twice that with a second gradient) or written, a few operations each.  Of 6551 GB/s:
// loss, 65 536 tokens of 2048 leaves 84.4 to 86 us (95 to 97 %); its gradient, 16 411 of 2048 24.5 us (84 %); back to the logits, 50 432
// tokens of 256 leaves 28.4 to 29 us (80 to 82 %), where issue slots count as well: some 25 instructions per node.
#pragma once

#include <float.h>

#include "common.cuh"

namespace fff {

// ---- balance loss ----------------------------------------------------------------------------------

constexpr int kBalThreads = 512;
constexpr int kBalCols = 128;                 // columns (leaves) per tile: few slices to add up (512: 35 us instead of 31 for 32 768 tokens of 512)
constexpr int kBalGroup = 16;                 // slices that a thread of the CTA that adds them up reads of its column
// Row slices per tile: two CTAs per SM.
__host__ inline int balance_max_slices(int tiles) { return tiles < 296 ? 296 / tiles : 1; }
// Slices that one CTA adds up: it has kBalThreads / cols threads per column.
__host__ __device__ inline int balance_group(int cols) { return kBalGroup * (kBalThreads / cols); }
__host__ __device__ inline int balance_groups(int slices, int cols) { return (slices + balance_group(cols) - 1) / balance_group(cols); }

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

// How tokens are told and counted.  kBalFew: at most 32 leaves, whose tokens every thread counts for its columns.  kBalRows: a row of a tile
// is a warp's; a lane looks at a row each, and rows that all count are added without asking (54 instructions per vector otherwise; 65 536
// tokens of 2048 leaves, with launch, 105 and 100 us).
enum : int { kBalFew = 0, kBalMany = 1, kBalRows = 2 };

// Grid (slices, tiles).  Every CTA adds up its rows of its columns and counts its rows' leaves among them; the last CTA of a tile
// adds up the slices in their order, the last tile the tiles: one launch, and the same bits every time.
// V: columns per thread (4; 1 for one or two leaves).  kHow: see above.  Rows are added in float32, 256 of a thread's at a time and then those sums (n rows: at
// most 256 + n / 256 roundings), then the threads of a column (at most 25 more); slices in float64.  (64 registers for two CTAs per SM; the
// form for 64 leaves spills 32 bytes.)
template <int V, int kHow>
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

    float* own = s_sum + (r * across + c) * V;            // [down][cols]
    float acc[V];
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = own[v] = 0.0f;
    int mine = 0, here[V];                                // rows; those of the thread's leaves (few leaves)
#pragma unroll
    for (int v = 0; v < V; ++v) here[v] = 0;
    const float* base = mix + col0 + c * V;
    for (int64_t block = b0 + r; block < b1; block += (int64_t)256 * down) {
        for (int64_t b = block; b < min(b1, block + (int64_t)256 * down); b += (int64_t)U * down) {
            if constexpr (kHow == kBalRows) {
                const int lane = tid & 31, last = (int)min(b1 - 1 - b, (int64_t)U * down);
                const TokenFlags own_row = token_flags(leaf_idx, mask, b + min((lane & (U - 1)) * down, last));
                const float* p = base + b * n_leaves;
                float4 q[U];
#pragma unroll
                for (int u = 0; u < U; ++u) q[u] = __ldcs(reinterpret_cast<const float4*>(p + (int64_t)min(u * down, last) * n_leaves));
                const bool ok = lane < U && lane * down <= last && own_row.counts(n_leaves);
                const unsigned in = __ballot_sync(kFullMask, ok);
                if (ok && (unsigned)(own_row.leaf - col0) < (unsigned)cols) atomicAdd(&s_hist[own_row.leaf - col0], 1);
                mine += __popc(in);
                if (in == (1u << U) - 1) {
#pragma unroll
                    for (int u = 0; u < U; ++u) { acc[0] += q[u].x; acc[1] += q[u].y; acc[2] += q[u].z; acc[3] += q[u].w; }
                } else {
                    // (rows that do not count are left out, not multiplied by zero: they may hold anything)
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (in >> u & 1) { acc[0] += q[u].x; acc[1] += q[u].y; acc[2] += q[u].z; acc[3] += q[u].w; }
                }
            } else {
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
#pragma unroll
                    for (int v = 0; v < V; ++v) acc[v] += in ? m[u][v] : 0.0f;
                    mine += in;
                    if constexpr (kHow == kBalFew) {
#pragma unroll
                        for (int v = 0; v < V; ++v) here[v] += in && flags[u].leaf == c * V + v;
                    } else if (c == 0 && in && (unsigned)(flags[u].leaf - col0) < (unsigned)cols) {
                        atomicAdd(&s_hist[flags[u].leaf - col0], 1);
                    }
                }
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) { own[v] += acc[v]; acc[v] = 0.0f; }
    }
    if (c != 0) mine = 0;
    mine = __reduce_add_sync(kFullMask, mine);
    if ((tid & 31) == 0 && mine) atomicAdd(&s_rows, mine);
    if constexpr (kHow == kBalFew) {                                             // (an atomic per token on eight words: 6 us for 2048 tokens)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            for (int o = across; o < 32; o <<= 1) here[v] += __shfl_xor_sync(kFullMask, here[v], o);
            if ((tid & 31) < across && here[v]) atomicAdd(&s_hist[c * V + v], here[v]);
        }
    }
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
    const int groups = balance_groups(slices, cols), group = blockIdx.x / balance_group(cols), first = group * balance_group(cols);
    const int members = min(balance_group(cols), slices - first);
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
    // what the threads of a column have, in the column's first (those of a warp first, where it has several)
    auto add_columns = [&](int of) {
        for (int o = cols; o < 32; o <<= 1) {
            sum += __shfl_xor_sync(kFullMask, sum, o);
            cnt += __shfl_xor_sync(kFullMask, cnt, o);
        }
        if (cols >= 32 || (tid & 31) < cols) {
            s_col[(cols < 32 ? tid >> 5 : r2) * cols + i] = sum;
            s_cnt[(cols < 32 ? tid >> 5 : r2) * cols + i] = cnt;
        }
        __syncthreads();
        if (tid < cols)
            for (int k = 1; k < (cols < 32 ? parts : min(each, of)); ++k) {
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
constexpr int kSlopeCols = 512;               // columns per tile

// Tokens that count: the sum of the counts (all of which belong to such tokens).  By all threads of a CTA.  (Counts are read as vectors,
// several in flight: one by one, four thousand took a CTA 8 us.)
__device__ __forceinline__ double counted_tokens(const int32_t* __restrict__ counts, int n_leaves, long long* s_red) {
    const int tid = threadIdx.x;
    long long n = 0;
    if ((reinterpret_cast<uintptr_t>(counts) & 15) == 0 && n_leaves >= 4) {
#pragma unroll 4
        for (int j = tid; j < n_leaves >> 2; j += blockDim.x) {
            const int4 q = __ldg(reinterpret_cast<const int4*>(counts) + j);
            n += (long long)q.x + q.y + (long long)q.z + q.w;
        }
    } else {
#pragma unroll 4
        for (int j = tid; j < n_leaves; j += blockDim.x) n += __ldg(counts + j);
    }
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
    const int cols = min(n_leaves, kSlopeCols), col0 = blockIdx.y * cols;
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
constexpr int kRoutePerSm = 2;                // CTAs per SM
constexpr int kRouteWarps = kRouteThreads / 32;
constexpr int kRouteChunk = 512;              // leaves that one warp reduces at a time: four per lane and four times that, nine levels
constexpr int kRouteMaxSlopeLeaves = 8192;    // trees whose slopes lie in shared memory (8192 leaves, 4096 tokens, from a table: 79 us instead of 74)

// Rows of up to a chunk are a warp's, as many at a time as make 512 weights; longer ones a CTA's, a chunk for every warp, several rows
// at a time where that takes them (one where the batch is short).  (Rows of 2048 by single warps: 78 us instead of 72, 16 384 tokens.)
struct RouteShape {
    int n_leaves, rows;
    bool balance;
    __host__ __device__ bool by_warps() const { return n_leaves <= kRouteChunk; }
    __host__ __device__ bool near_slopes() const { return n_leaves <= kRouteMaxSlopeLeaves; }
    // Floats of shared memory: sums of the chunks (two groups' in turn), slopes.
    __host__ __device__ int top() const { return by_warps() ? 0 : 2 * rows * (n_leaves / kRouteChunk); }
    __host__ __device__ int slopes() const { return balance && near_slopes() ? n_leaves : 0; }
    __host__ __device__ size_t bytes() const { return sizeof(float) * (size_t)(2 * top() + slopes()); }
};
__host__ inline RouteShape route_shape(int64_t B, int n_leaves, bool balance, int sms) {
    if (n_leaves <= kRouteChunk) return {n_leaves, kRouteChunk / n_leaves, balance};
    const int rows = kRouteWarps * kRouteChunk / n_leaves;
    return {n_leaves, rows < 1 || B < (int64_t)sms * rows ? 1 : rows, balance};
}

// One node: sums over its two children's leaves in, its own out.  Children too small for float32 have no say.
__device__ __forceinline__ float node_gradient(float ml, float sl, float mr, float sr, float& m, float& s) {
    m = ml + mr;
    s = sl + sr;
    const float inv = rcp_approx(m);
    const float g = sr * (ml * inv) - sl * (mr * inv);
    return m < FLT_MIN ? 0.0f : g;
}

// A lane's part of up to 512 mixture weights and what belongs to them: four neighbouring leaves of each of four chunks of 128.  D is the
// depth, 9 for every one from 9 on (512 weights are then a row's, or a part of one's): with it known, indices are constants but for the
// lane, and the kernel, which issue bounds, has 40 % fewer instructions.
constexpr int kRouteU = 4;
constexpr int kRouteDeepest = 9;
template <int D>
struct RouteIn {
    static constexpr int kRows = D >= 9 ? 1 : D == 8 ? 2 : kRouteU;      // rows that the four chunks are of
    static constexpr int row_of(int i) { return i * kRows / kRouteU; }
    float m[kRouteU][4], g[kRouteU][4];
    int leaf[kRows], kept[kRows];                          // of the lane's rows (not at depth 1)
};

// Loads them: `base` on from row row0, whose group of rows ends at `elems`.  What lies behind the end is some of the last row instead
// (loads without branches; nothing of it is stored).
template <bool kUp, bool kBal, int D>
__device__ __forceinline__ void route_load(const float* __restrict__ mix, const float* __restrict__ dmix, const int32_t* __restrict__ leaf_idx,
                                           const uint8_t* __restrict__ mask, int64_t row0, int base, int elems, int depth, int lane, RouteIn<D>& in)
{
    const float* gm = mix + (row0 << depth);
    const float* gd = kUp ? dmix + (row0 << depth) : nullptr;
#pragma unroll
    for (int i = 0; i < kRouteU; ++i) {
        int e = base + i * 128 + lane * 4;
        if constexpr (D == 1) {                            // (a lane's four weights are two rows, and the last lane may have one)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                in.m[i][k] = e + k < elems ? gm[e + k] : 0.0f;
                in.g[i][k] = kUp && e + k < elems ? gd[e + k] : 0.0f;
            }
        } else {
            if constexpr (D < 9) e = min(e, elems - 4);
            if (i == 0 || in.row_of(i) != in.row_of(i - 1)) {
                const int64_t b = row0 + (e >> depth);
                in.leaf[in.row_of(i)] = kBal && leaf_idx ? __ldg(leaf_idx + b) : 0;
                in.kept[in.row_of(i)] = mask ? __ldg(mask + b) : 1;
            }
            const float4 q = __ldcs(reinterpret_cast<const float4*>(gm + e));
            in.m[i][0] = q.x; in.m[i][1] = q.y; in.m[i][2] = q.z; in.m[i][3] = q.w;
            const float4 d = kUp ? __ldcs(reinterpret_cast<const float4*>(gd + e)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            in.g[i][0] = d.x; in.g[i][1] = d.y; in.g[i][2] = d.z; in.g[i][3] = d.w;
        }
    }
}

// Where the gradients of such weights go: to rows from `out` on, dense.
template <int D>
struct RouteOut {
    float* out;                                            // D = 9: the row
    int depth, at, elems;                                  // weights: first (D = 9: of the row), how many
    // the node 2^(2 + k) leaves wide that leaf w of them belongs to (k = -1: the first of two)
    __device__ __forceinline__ float* node(int w, int k) const {
        if constexpr (D >= 9) return out + ((1 << (depth - 2 - k)) - 1 + (at >> (2 + k))) + (w >> (2 + k));
        else return out + (w >> D) * ((1 << D) - 1) + (1 << (D - 2 - k)) - 1 + ((w & ((1 << D) - 1)) >> (2 + k));
    }
    __device__ __forceinline__ void store(int w, int k, float g) const {
        if (D >= 9 || w < elems) *node(w, k) = g;
    }
};

// Two levels, in a lane's registers; m, t: the sums over its four leaves of every chunk.  slope: of the lane's leaves (D <= 7: the same
// ones in every chunk), else slopes has them.  A row that the mask leaves out has weights of zero, which give zeros whatever its
// gradients are.
template <bool kBal, int D>
__device__ __forceinline__ void route_low(RouteIn<D>& in, const int32_t* __restrict__ leaf_idx, const uint8_t* __restrict__ mask,
                                          const float* slopes, float4 slope, int64_t row0, const RouteOut<D>& to, int lane,
                                          float (&m)[kRouteU], float (&t)[kRouteU])
{
    const int L = D >= 9 ? 1 << to.depth : 1 << D;
#pragma unroll
    for (int i = 0; i < kRouteU; ++i) {
        const int e = i * 128 + lane * 4;
        float (&w)[4] = in.m[i], (&d)[4] = in.g[i];
        if constexpr (D == 1) {
#pragma unroll
            for (int k = 0; k < 4; k += 2) {
                if (e + k >= to.elems) break;
                const int64_t b = row0 + ((e + k) >> 1);
                if (kBal && (!leaf_idx || (unsigned)__ldg(leaf_idx + b) < 2u)) { d[k] += slope.x; d[k + 1] += slope.y; }
                if (mask && __ldg(mask + b) == 0) w[k] = w[k + 1] = 0.0f;
            }
        } else {
            if (kBal && (unsigned)in.leaf[in.row_of(i)] < (unsigned)L) {
                const float4 q = D <= 7 ? slope : *reinterpret_cast<const float4*>(slopes + (D == 8 ? e & 255 : to.at + e));
                d[0] += q.x; d[1] += q.y; d[2] += q.z; d[3] += q.w;
            }
            if (!in.kept[in.row_of(i)]) w[0] = w[1] = w[2] = w[3] = 0.0f;
        }
        float ma, sa, mb, sb;
        const float g0 = node_gradient(w[0], w[0] * d[0], w[1], w[1] * d[1], ma, sa);
        const float g1 = node_gradient(w[2], w[2] * d[2], w[3], w[3] * d[3], mb, sb);
        if constexpr (D == 1) {
            if (e < to.elems) to.out[e >> 1] = g0;
            if (e + 2 < to.elems) to.out[(e >> 1) + 1] = g1;
        } else {
            const float g2 = node_gradient(ma, sa, mb, sb, m[i], t[i]);
            if (D >= 9 || e < to.elems) {
                float* last = to.node(e, -1);
                last[0] = g0;
                last[1] = g1;
                *to.node(e, 0) = g2;
            }
        }
    }
}

// The levels above: up to five across the lanes, the chunks shared out on the way: after the first step a lane goes on with two of the
// four, after the second with one, so that a level costs what its nodes do (every lane going on with all four: 20 nodes and 40 shuffles
// instead of 6 and 12); then up to two across the chunks.  mm, ss: the sums over all 512.
template <int D>
__device__ __forceinline__ void route_high(const float (&m)[kRouteU], const float (&t)[kRouteU], const RouteOut<D>& to, int lane, float& mm, float& ss)
{
    const bool r0 = lane & 1, r1 = lane & 2;
    mm = ss = 0.0f;
    if constexpr (D >= 3) {
        float m2[2], t2[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            // chunk i stays with even lanes, chunk 2 + i with odd ones
            const float mo = __shfl_xor_sync(kFullMask, r0 ? m[i] : m[2 + i], 1), so = __shfl_xor_sync(kFullMask, r0 ? t[i] : t[2 + i], 1);
            const float mk = r0 ? m[2 + i] : m[i], sk = r0 ? t[2 + i] : t[i];
            const float g = node_gradient(r0 ? mo : mk, r0 ? so : sk, r0 ? mk : mo, r0 ? sk : so, m2[i], t2[i]);
            to.store((lane & 1) * 256 + i * 128 + (lane & ~1) * 4, 1, g);
        }
        if constexpr (D >= 4) {
            const int mine = (lane & 1) * 256 + (lane & 2) * 64;         // first leaf of the chunk that the lane goes on with
            {
                const float mo = __shfl_xor_sync(kFullMask, r1 ? m2[0] : m2[1], 2), so = __shfl_xor_sync(kFullMask, r1 ? t2[0] : t2[1], 2);
                const float mk = r1 ? m2[1] : m2[0], sk = r1 ? t2[1] : t2[0];
                const float g = node_gradient(r1 ? mo : mk, r1 ? so : sk, r1 ? mk : mo, r1 ? sk : so, mm, ss);
                to.store(mine + (lane & ~3) * 4, 2, g);
            }
            auto up = [&](int lanes, bool right) {         // one more level: with the lane that has the other child
                const float mo = __shfl_xor_sync(kFullMask, mm, lanes), so = __shfl_xor_sync(kFullMask, ss, lanes);
                return node_gradient(right ? mo : mm, right ? so : ss, right ? mm : mo, right ? ss : so, mm, ss);
            };
#pragma unroll
            for (int k = 3; k <= 5; ++k) {
                if (k > D - 2) break;
                const float g = up(1 << (k - 1), (lane >> (k - 1)) & 1);
                if (((lane >> 2) & ((1 << (k - 2)) - 1)) == 0) to.store(mine + (lane & ~((1 << k) - 1)) * 4, k, g);
            }
            // chunks 0 and 1, 2 and 3; then both pairs
            if constexpr (D >= 8) {
                const float g = up(2, r1);
                if ((lane & ~1) == 0) to.store(mine, 6, g);
            }
            if constexpr (D >= 9) {
                const float g = up(1, r0);
                if (lane == 0) to.store(0, 7, g);
            }
        }
    }
}

// kUp: dmixture given; kBal: counts and dloss given (slope_table for more than kRouteMaxSlopeLeaves leaves).
// Gradients are stored as they come: a row has 2^d - 1 of them and starts anywhere, a level's are next to each other, L2 puts them
// together.  (Collected in shared memory, and stored as aligned vectors: the same times, 5 % more at 2048 leaves.)
template <bool kUp, bool kBal, int D>
__global__ void __launch_bounds__(kRouteThreads, kRoutePerSm)
k_routing_backward(const float* __restrict__ mix, const float* __restrict__ dmix, const int32_t* __restrict__ leaf_idx,
                   const uint8_t* __restrict__ mask, const int32_t* __restrict__ counts, const float* __restrict__ dloss,
                   const float* __restrict__ slope_table, float* __restrict__ dz, int64_t B, int any_depth, const RouteShape S)
{
    extern __shared__ __align__(16) float s_route[];
    __shared__ long long s_red[kRouteWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int depth = D < kRouteDeepest ? D : any_depth, L = 1 << depth, N = L - 1, R = S.rows, chunks = L / kRouteChunk;
    const bool by_warps = D < kRouteDeepest || chunks == 1;
    float* s_slope = s_route;                                            // [L]
    float* s_top = s_route + S.slopes();                                 // [2 groups][2][R][chunks]
    const float* slopes = S.near_slopes() ? s_slope : slope_table;
    pdl_trigger();
    pdl_wait();
    const int64_t groups = (B + R - 1) / R;
    int64_t grp = by_warps ? (int64_t)blockIdx.x + (int64_t)gridDim.x * warp : blockIdx.x;
    const int64_t stride = by_warps ? (int64_t)gridDim.x * kRouteWarps : gridDim.x;
    const int from = by_warps ? 0 : warp, step = by_warps ? 1 : kRouteWarps;
    auto elems_of = [&](int64_t group) { return (int)min((int64_t)R, B - group * R) * L; };
    // a warp's next 512 weights are on their way while it works on the upper levels of these
    RouteIn<D> in;
    auto load = [&](int64_t group, int u) {
        if (group < groups && u * kRouteChunk < elems_of(group))         // (a short row has none for some warps)
            route_load<kUp, kBal, D>(mix, dmix, leaf_idx, mask, group * R, u * kRouteChunk, elems_of(group), depth, lane, in);
    };
    load(grp, from);
    float4 slope = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (kBal && S.near_slopes()) {
        const double n = counted_tokens(counts, L, s_red), g = slope_scale(dloss, n);
#pragma unroll 4
        for (int j = tid; j < L; j += kRouteThreads) s_slope[j] = centred_slope(__ldg(counts + j), L, n, g);
        __syncthreads();
        if constexpr (D <= 7) {
            const float* at = s_slope + (lane * 4 & (L - 1));
            slope = D == 1 ? make_float4(at[0], at[1], 0.0f, 0.0f) : *reinterpret_cast<const float4*>(at);
        }
    }
    for (int turn = 0; grp < groups; grp += stride, turn ^= 1) {
        const int64_t row0 = grp * R;
        const int elems = elems_of(grp), rows = elems >> depth;
        float* out = dz + row0 * N;
        float* top = s_top + turn * S.top();
        for (int u = from; u * kRouteChunk < elems; u += step) {
            const int base = u * kRouteChunk;
            RouteOut<D> nodes{out, depth, 0, elems};
            if constexpr (D >= kRouteDeepest) {
                nodes.out = out + (int64_t)(base >> depth) * N;
                nodes.at = base & (L - 1);
            }
            float m[kRouteU], t[kRouteU], mm, ss;
            route_low<kBal, D>(in, leaf_idx, mask, slopes, slope, row0, nodes, lane, m, t);
            const bool more = (u + step) * kRouteChunk < elems;
            load(more ? grp : grp + stride, more ? u + step : from);
            route_high<D>(m, t, nodes, lane, mm, ss);
            if (!by_warps && lane == 0) {
                top[u] = mm;                                             // u = row * chunks + chunk
                top[R * chunks + u] = ss;
            }
        }
        if (by_warps) continue;
        // The levels above the chunks: a warp per row, in place (a step's reads lie ahead of its writes).  One barrier per group: the other
        // warps go on to the next, whose sums have another place.
        __syncthreads();
        for (int row = warp; row < rows; row += kRouteWarps) {
            float* tm = top + row * chunks;
            float* ts = tm + R * chunks;
            float* o = out + (int64_t)row * N;
            for (int nodes = chunks >> 1; nodes >= 1; nodes >>= 1) {
                for (int p0 = 0; p0 < nodes; p0 += 32) {
                    const int p = p0 + lane;
                    float mm, ss;
                    if (p < nodes) o[nodes - 1 + p] = node_gradient(tm[2 * p], ts[2 * p], tm[2 * p + 1], ts[2 * p + 1], mm, ss);
                    __syncwarp();
                    if (p < nodes) { tm[p] = mm; ts[p] = ss; }
                    __syncwarp();
                }
            }
        }
    }
}

}  // namespace fff
