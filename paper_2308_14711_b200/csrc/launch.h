// How the launchers outside fff_api.cu start their kernels, and what they take.  (fff_api.cu checks arguments, owns all memory and
// calls these; a launcher only enqueues.)
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace fff {

struct LaunchOn {
    cudaStream_t stream;
    int device, sm_count;
    bool dependent;               // as a programmatic dependent launch: every kernel waits (pdl_wait) before its first access to anything that
                                  // a kernel may have written (the weights of a handle are never written again, and may be read before)
};

template <typename... KArgs, typename... Args>
cudaError_t launch_on(const LaunchOn& on, void (*kern)(KArgs...), unsigned grid_x, unsigned grid_y, unsigned block, size_t smem, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid_x, grid_y);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = on.stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = on.dependent ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

// ---- routing.cu: the routing losses -----------------------------------------------------------------

// Fixed scratch of a handle for balance_loss: sized by the number of leaves alone, its counters zero between calls.
size_t balance_scratch_bytes(int64_t n_leaves);

// The part of it that routing_backward may use for the slopes (L floats).
float* balance_scratch_slope(void* scratch, int64_t n_leaves);

// mixture [B, L], leaf_idx [B], mask [B] or nullptr; loss [1], counts [L], mean [L], each may be nullptr.
cudaError_t balance_loss(const LaunchOn& on, const float* mixture, const int32_t* leaf_idx, const uint8_t* mask, float* loss,
                         int32_t* counts, float* mean, int64_t B, int64_t n_leaves, void* scratch);

cudaError_t balance_loss_backward(const LaunchOn& on, const int32_t* leaf_idx, const uint8_t* mask, const int32_t* counts,
                                  const float* dloss, float* dmixture, int64_t B, int64_t n_leaves);

// counts == nullptr: no balance loss.  slope: scratch of L floats.
cudaError_t routing_backward(const LaunchOn& on, const float* mixture, const float* dmixture, const int32_t* leaf_idx,
                             const uint8_t* mask, const int32_t* counts, const float* dloss, float* dlogits, int64_t B, int depth,
                             float* slope, int* launches);

// ---- mx4.cu: microscaled 4-bit weights --------------------------------------------------------------

// elem_bytes: 4 float32, 2 bf16; values may be nullptr.
cudaError_t quantize_mx4(const LaunchOn& on, const void* src, int elem_bytes, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales,
                         void* values);
cudaError_t dequantize_mx4(const LaunchOn& on, const uint8_t* codes, const uint8_t* scales, int elem_bytes, int64_t rows, int64_t cols,
                           void* values);

// A layer's image (owned by its handle).
struct Mx4Layer {
    unsigned char* image = nullptr;
    int D = 0, O = 0, l = 0;
    bool mma = false;             // leaves wide enough for the tensor-core kernel
    bool big = false;             // some scale is over 2
};
bool mx4_on_tensor_cores(int leaf_width);
constexpr int kMx4MaxLeafWidth = 1024;           // hidden values of a tile are kept in shared memory
size_t mx4_image_bytes(const Mx4Layer& m, int64_t n_leaves);
bool mx4_record_fits(const Mx4Layer& m);          // offsets inside a leaf's record are ints
// flag: one int of device memory, zero; set where a scale is over 2.
cudaError_t mx4_find_big(const uint8_t* scales, int64_t n, int* flag, int sm_count);
cudaError_t mx4_pack(const Mx4Layer& m, const uint8_t* w1, const uint8_t* s1, const uint8_t* w2, const uint8_t* s2, const void* b1,
                     const void* b2, int64_t n_leaves, int sm_count);

// The leaf kernels.  tiles / n_tiles: a tile list over perm; counts != nullptr: perm is the table of lists [n_leaves][cap] instead.
struct Mx4Tokens {
    const void *x;
    void *y;
    int act;
    int* status;
    int x_cols = 0;               // mx4_tokens: row length of x, the layer's or up to seven less
};
// The other kernels want rows of x that are 16-byte vectors, and store rows of y fastest that are.  Copies rows of bf16 values to rows of
// another length (both buffers on 16-byte boundaries): what a longer row has more is zero.
cudaError_t mx4_copy_rows(const LaunchOn& on, void* dst, int dst_cols, const void* src, int src_cols, int64_t rows);
// Rows of the largest tile worth having; lists of up to n_leaves leaves.
int mx4_most_rows(const Mx4Layer& m, int n_leaves);
cudaError_t mx4_leaf_tiles(const LaunchOn& on, const Mx4Layer& m, const Mx4Tokens& t, const int32_t* perm, const void* tiles, int n_tiles,
                           int tile_rows, int32_t* counts, int n_leaves, int cap);
// A few tokens: the walk and the leaf in one launch, a CTA per token.
bool mx4_token_fits(const Mx4Layer& m);
cudaError_t mx4_tokens(const LaunchOn& on, const Mx4Layer& m, const Mx4Tokens& t, const void* node_w, const void* node_b, int depth, int32_t* leaf_out,
                       int32_t* leaf_out2, int64_t B);
// The tail of the walk (levels > 0) as in k_leaf_warp.
struct Mx4Tail {
    const void *node_w = nullptr, *node_b = nullptr;
    int level0 = 0, levels = 0;
    const int32_t* pos = nullptr;
    int32_t* leaf_out = nullptr;
};
cudaError_t mx4_leaf_rows(const LaunchOn& on, const Mx4Layer& m, const Mx4Tokens& t, const int32_t* leaf_idx, const int32_t* perm, int64_t B,
                          const Mx4Tail& tail);

}  // namespace fff
