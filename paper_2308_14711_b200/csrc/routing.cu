// Launchers of the routing losses (kernels/routing.cuh); arguments are checked by their callers in fff_api.cu.
#include "kernels/routing.cuh"

#include <algorithm>
#include <mutex>

#include "launch.h"

namespace fff {

namespace {

constexpr int kMaxDevices = 64;

int balance_tiles(int64_t n_leaves) { return (int)std::max<int64_t>(1, n_leaves / kBalCols); }

// Slices so that every thread of a CTA has a few rows to add up; one where the whole batch is little more than that.
int slices_for(int64_t B, int64_t n_leaves, int threads, int rows_each, int most) {
    const int64_t cols = std::min<int64_t>(n_leaves, kBalCols), down = threads / (cols >= 4 ? cols / 4 : cols);
    return (int)std::max<int64_t>(1, std::min<int64_t>(most, (B + down * rows_each - 1) / (down * rows_each)));
}

BalanceScratch layout(void* scratch, int64_t n_leaves) {
    const size_t T = balance_tiles(n_leaves), S = balance_max_slices((int)T), G = balance_groups((int)S);
    BalanceScratch ws;
    ws.loss = static_cast<double*>(scratch);
    ws.group_sums = ws.loss + ((T + 1) & ~(size_t)1);      // (the rest starts on a 16-byte boundary)
    ws.parts = reinterpret_cast<float2*>(ws.group_sums + ((G * n_leaves + 1) & ~(size_t)1));
    ws.group_counts = reinterpret_cast<int32_t*>(ws.parts + S * n_leaves);
    ws.rows = ws.group_counts + G * n_leaves;
    ws.group_rows = ws.rows + S * T;
    ws.done = ws.group_rows + G * T;
    return ws;
}

}  // namespace

float* balance_scratch_slope(void* scratch, int64_t n_leaves) {
    return reinterpret_cast<float*>(layout(scratch, n_leaves).parts);
}

size_t balance_scratch_bytes(int64_t n_leaves) {
    const size_t T = balance_tiles(n_leaves), S = balance_max_slices((int)T), G = balance_groups((int)S);
    return 8 * (T + 1) + 8 * (G * n_leaves + 1) + 8 * S * n_leaves + 4 * (G * n_leaves + S * T + G * T + T * (G + 1) + 1);
}

cudaError_t balance_loss(const LaunchOn& on, const float* mixture, const int32_t* leaf_idx, const uint8_t* mask, float* loss,
                         int32_t* counts, float* mean, int64_t B, int64_t n_leaves, void* scratch) {
    const int S = slices_for(B, n_leaves, kBalThreads, 8, balance_max_slices(balance_tiles(n_leaves)));
    const unsigned T = (unsigned)balance_tiles(n_leaves);
    return launch_on(on, n_leaves >= 4 ? k_balance_loss<4> : k_balance_loss<1>, (unsigned)S, T, kBalThreads, 0, mixture, leaf_idx, mask, loss,
                     counts, mean, B, (int)n_leaves, layout(scratch, n_leaves));
}

cudaError_t balance_loss_backward(const LaunchOn& on, const int32_t* leaf_idx, const uint8_t* mask, const int32_t* counts,
                                  const float* dloss, float* dmixture, int64_t B, int64_t n_leaves) {
    const unsigned T = (unsigned)balance_tiles(n_leaves);
    const int most = std::max(1, on.sm_count * 4 / (int)T);
    const int S = slices_for(B, n_leaves, kSlopeThreads, 4, most);
    return launch_on(on, n_leaves >= 4 ? k_balance_loss_backward<4> : k_balance_loss_backward<1>, (unsigned)S, T, kSlopeThreads, 0, leaf_idx,
                     mask, counts, dloss, dmixture, B, (int)n_leaves);
}

cudaError_t routing_backward(const LaunchOn& on, const float* mixture, const float* dmixture, const int32_t* leaf_idx,
                             const uint8_t* mask, const int32_t* counts, const float* dloss, float* dlogits, int64_t B, int depth,
                             float* slope, int* launches) {
    const int L = 1 << depth;
    const bool up = dmixture != nullptr, bal = counts != nullptr;
    *launches = 0;
    if (bal && !route_staged(L)) {
        const cudaError_t e = launch_on(on, k_balance_slope, (unsigned)std::min(on.sm_count, L / 1024), 1, 1024, 0, counts, dloss, slope, L);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    const auto kern = up ? (bal ? k_routing_backward<true, true> : k_routing_backward<true, false>) : k_routing_backward<false, true>;
    const size_t smem = RouteSmem{L, bal}.bytes();
    const int which = up ? (bal ? 0 : 1) : 2;
    if (smem > 48 * 1024) {
        static std::mutex mu;
        static bool raised[3][kMaxDevices] = {};
        std::lock_guard<std::mutex> lk(mu);
        if (!raised[which][on.device]) {
            const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
            if (e != cudaSuccess) return e;
            raised[which][on.device] = true;
        }
    }
    const int64_t groups = (B + route_rows(L) - 1) / route_rows(L);
    const int per_sm = (int)std::max<size_t>(1, std::min<size_t>(kRoutePerSm, (size_t)(227 * 1024) / (smem + 1024)));
    const int64_t ctas = route_by_warps(L) ? (groups + kRouteWarps - 1) / kRouteWarps : groups;
    // (a batch that would not give every SM a CTA: a warp of work each)
    const unsigned grid = (unsigned)std::min<int64_t>(ctas < on.sm_count ? groups : ctas, (int64_t)on.sm_count * per_sm);
    const cudaError_t e = launch_on(on, kern, grid, 1, kRouteThreads, smem, mixture, dmixture, leaf_idx, mask, counts, dloss,
                                    (const float*)slope, dlogits, B, depth);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace fff
