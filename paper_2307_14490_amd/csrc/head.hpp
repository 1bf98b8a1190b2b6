// Internal declarations of the softmax head's operators: layer norm, the exact
// softmax loss and AdamW (host layer: api_head.hip).
#pragma once

#include "common.hpp"

namespace huge {

// ---------------------------------------------------------------------------
// Layer norm (k_norm.hip)
// ---------------------------------------------------------------------------
constexpr int kNormMaxDim = 8192;
constexpr int kNormBlocks = 1024;  // workgroups of the backward pass, at most: the rows of
                                   // partial weight gradients that are summed at the end
struct NormArgs {
    const void* x;
    const void* dy;   // backward pass only
    void* y;          // y, or dx (backward pass; may be null)
    int64_t ld_x, ld_dy, ld_y, n;
    int32_t dim, dtype;
    const float* gamma;
    const float* beta;
    float eps;
    float* mean;
    float* rstd;
    float* partial;   // backward pass: [workgroups][2][dim], or null
    bool vec;         // four elements at a time
};
int norm_blocks(int64_t n, int32_t dim);
hipError_t launch_norm(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, float* dgamma, float* dbeta, hipStream_t s);

// ---------------------------------------------------------------------------
// AdamW (k_adamw.hip)
// ---------------------------------------------------------------------------
constexpr int kAdamTensors = 64;    // tensors of a launch
constexpr int kAdamBlock = 256;     // elements that share the scales of an 8-bit state
constexpr int kAdamChunk = 4096;    // elements of a workgroup
constexpr int64_t kAdamMaxElements = (int64_t)1 << 40;

struct AdamTensor {
    void* p;
    const void* g;
    uint8_t* state;
    int64_t n;
    uint32_t first;   // its first chunk among the launch's
    uint32_t vec;     // p, g (or m, v) aligned for four elements at a time
};
struct AdamArgs {
    AdamTensor t[kAdamTensors];
    int32_t count;
    float beta1, one_beta1, beta2, one_beta2, rate, fix, eps, keep, grad_scale;
    int32_t* status;
};
// Offsets in a state: m, then v, then (8 bits) the two scales of each block.
__host__ __device__ inline int64_t adam_padded(int64_t n) {
    return (n + kAdamBlock - 1) / kAdamBlock * kAdamBlock;
}
hipError_t launch_adamw(const AdamArgs& a, int64_t chunks, int32_t p_dtype, int32_t g_dtype,
                        int32_t state_kind, hipStream_t s);
// p: m, g: v of AdamTensor, as floats
hipError_t launch_adamw_state(const AdamArgs& a, int64_t chunks, int32_t state_kind, bool write,
                              hipStream_t s);

// ---------------------------------------------------------------------------
// Exact softmax loss (k_softmax.hip)
// ---------------------------------------------------------------------------
// Rows are packed in records of kSmTile, as the operands of 32x32x16 matrix
// products in the order in which a wave's lanes take them.
constexpr int kSmTile = 32;
constexpr int64_t kSmPieceBytes = (int64_t)2 << 30;  // packed table rows, at most
constexpr int64_t kSmPartRows = 131072;              // rows of partial sums of a pass

// How a call of n rows is laid out, from its sizes alone.
struct SoftmaxPlan {
    int32_t dim, parts, nd, chunks, dp, kd;  // nd 32-wide blocks of dp in each of `chunks`
    int64_t classes;
    int64_t piece;                           // classes packed together (multiple of kSmTile)
    int64_t rows_pad;                        // n in whole tiles
    size_t h, w, part, row_part, total;      // workspace offsets
};
SoftmaxPlan softmax_plan(int64_t classes, int64_t n, int32_t dim, int32_t dtype, bool grad);

struct SoftmaxArgs {
    const void* h;
    const void* w;
    int64_t ld_h, ld_w, n, classes;
    int32_t dim, dtype;
    const float* bias;
    const int32_t* labels;
    const float* weight;
    float* loss;          // forward
    float* lse;           // forward: written, backward: read
    double* loss_sum;
    float scale;          // backward
    void* dh;
    void* dw;
    float* dbias;
    int32_t* status;
    uint8_t* ws;
    bool vec, vec16;      // h and w can be read four elements, 16 bytes at a time
};
hipError_t launch_softmax_loss(const SoftmaxArgs& a, hipStream_t s);
hipError_t launch_softmax_grad(const SoftmaxArgs& a, hipStream_t s);

}  // namespace huge
