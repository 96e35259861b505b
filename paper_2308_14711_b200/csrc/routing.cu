// Launchers of the routing losses (kernels/routing.cuh); arguments are checked by their callers in fff_api.cu.
#include "kernels/routing.cuh"

#include <algorithm>
#include <type_traits>

#include "launch.h"

namespace fff {

namespace {

int balance_tiles(int64_t n_leaves, int cols = kBalCols) { return (int)std::max<int64_t>(1, n_leaves / cols); }

// Slices so that every thread of a CTA has a few rows to add up; one where the whole batch is little more than that.
int slices_for(int64_t B, int64_t cols, int threads, int rows_each, int most) {
    const int64_t down = threads / (cols >= 4 ? cols / 4 : cols);
    return (int)std::max<int64_t>(1, std::min<int64_t>(most, (B + down * rows_each - 1) / (down * rows_each)));
}

BalanceScratch layout(void* scratch, int64_t n_leaves) {
    const size_t T = balance_tiles(n_leaves), S = balance_max_slices((int)T), G = balance_groups((int)S, (int)std::min<int64_t>(n_leaves, kBalCols));
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
    const size_t T = balance_tiles(n_leaves), S = balance_max_slices((int)T), G = balance_groups((int)S, (int)std::min<int64_t>(n_leaves, kBalCols));
    return 8 * (T + 1) + 8 * (G * n_leaves + 1) + 8 * S * n_leaves + 4 * (G * n_leaves + S * T + G * T + T * (G + 1) + 1);
}

cudaError_t balance_loss(const LaunchOn& on, const float* mixture, const int32_t* leaf_idx, const uint8_t* mask, float* loss,
                         int32_t* counts, float* mean, int64_t B, int64_t n_leaves, void* scratch) {
    const int S = slices_for(B, std::min<int64_t>(n_leaves, kBalCols), kBalThreads, 8, balance_max_slices(balance_tiles(n_leaves)));
    const unsigned T = (unsigned)balance_tiles(n_leaves);
    return launch_on(on, n_leaves < 4 ? k_balance_loss<1, kBalFew> : n_leaves <= 32 ? k_balance_loss<4, kBalFew> :
                         n_leaves < kBalCols ? k_balance_loss<4, kBalMany> : k_balance_loss<4, kBalRows>, (unsigned)S, T, kBalThreads, 0, mixture, leaf_idx, mask, loss,
                     counts, mean, B, (int)n_leaves, layout(scratch, n_leaves));
}

cudaError_t balance_loss_backward(const LaunchOn& on, const int32_t* leaf_idx, const uint8_t* mask, const int32_t* counts,
                                  const float* dloss, float* dmixture, int64_t B, int64_t n_leaves) {
    const unsigned T = (unsigned)balance_tiles(n_leaves, kSlopeCols);
    const int most = std::max(1, on.sm_count * 4 / (int)T);
    const int S = slices_for(B, std::min<int64_t>(n_leaves, kSlopeCols), kSlopeThreads, 4, most);
    return launch_on(on, n_leaves >= 4 ? k_balance_loss_backward<4> : k_balance_loss_backward<1>, (unsigned)S, T, kSlopeThreads, 0, leaf_idx,
                     mask, counts, dloss, dmixture, B, (int)n_leaves);
}

cudaError_t routing_backward(const LaunchOn& on, const float* mixture, const float* dmixture, const int32_t* leaf_idx,
                             const uint8_t* mask, const int32_t* counts, const float* dloss, float* dlogits, int64_t B, int depth,
                             float* slope, int* launches) {
    const int L = 1 << depth;
    const bool up = dmixture != nullptr, bal = counts != nullptr;
    *launches = 0;
    const RouteShape shape = route_shape(B, L, bal, on.sm_count);
    if (bal && !shape.near_slopes()) {
        const cudaError_t e = launch_on(on, k_balance_slope, (unsigned)std::min(on.sm_count, L / 1024), 1, 1024, 0, counts, dloss, slope, L);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    const int64_t groups = (B + shape.rows - 1) / shape.rows;
    const int64_t ctas = shape.by_warps() ? (groups + kRouteWarps - 1) / kRouteWarps : groups;
    // (a batch that would not give every SM a CTA: a warp of work each)
    const unsigned grid = (unsigned)std::min<int64_t>(ctas < on.sm_count ? groups : ctas, (int64_t)on.sm_count * kRoutePerSm);
    const auto launch = [&](auto d) {
        constexpr int D = decltype(d)::value;
        const auto kern = up ? (bal ? k_routing_backward<true, true, D> : k_routing_backward<true, false, D>) : k_routing_backward<false, true, D>;
        return launch_on(on, kern, grid, 1, kRouteThreads, shape.bytes(), mixture, dmixture, leaf_idx, mask, counts, dloss, (const float*)slope,
                         dlogits, B, depth, shape);
    };
    cudaError_t e;
    switch (std::min(depth, kRouteDeepest)) {
    case 1: e = launch(std::integral_constant<int, 1>()); break;
    case 2: e = launch(std::integral_constant<int, 2>()); break;
    case 3: e = launch(std::integral_constant<int, 3>()); break;
    case 4: e = launch(std::integral_constant<int, 4>()); break;
    case 5: e = launch(std::integral_constant<int, 5>()); break;
    case 6: e = launch(std::integral_constant<int, 6>()); break;
    case 7: e = launch(std::integral_constant<int, 7>()); break;
    case 8: e = launch(std::integral_constant<int, 8>()); break;
    default: e = launch(std::integral_constant<int, kRouteDeepest>());
    }
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace fff
