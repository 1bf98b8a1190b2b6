// Internal declarations of the softmax head's operators: layer norm, the exact
// softmax loss and AdamW (host layer: api_head.hip); RMS norm, rows in 8 bits, log
// probabilities and clipped gradients (host layer: api_answer.hip).
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
// RMS norm and rows in 8 bits (k_rms.hip)
// ---------------------------------------------------------------------------
constexpr int kByteBlock = 32;     // columns that share a scale
constexpr int kByteLeast = -100;   // smallest exponent of one

struct RmsArgs {
    const void* x;     // backward pass: the normalised rows; from 8 bits: unused
    const void* res;   // the residual, or null; backward pass: the gradient of the sum
    const void* dy;    // backward pass only
    void* total;       // x + res
    void* y;           // y, or dx (backward pass; may be null), or the values of 8 bits
    uint8_t* codes;    // y in 8 bits
    uint8_t* scales;
    int64_t ld_x, ld_res, ld_dy, ld_total, ld_y, ld_codes, ld_scales, n;
    int32_t dim, dtype;
    const float* gamma;
    float eps;
    float* rstd;
    float* partial;    // backward pass: [workgroups][dim], or null
    bool vec;          // four elements at a time
    bool eights;       // eight: 16 bytes of bf16 rows, 8 of codes
};
hipError_t launch_rms(const RmsArgs& a, hipStream_t s);
hipError_t launch_rms_backward(const RmsArgs& a, float* dgamma, hipStream_t s);
hipError_t launch_to_bytes(const RmsArgs& a, hipStream_t s);
hipError_t launch_from_bytes(const RmsArgs& a, hipStream_t s);

#if defined(__HIPCC__)
// The power of two that a scale stands for: 127 + its exponent, 255 for NaN.
__device__ __forceinline__ float byte_scale(uint32_t b) {
    return __uint_as_float(b == 255u ? 0x7FC00000u : b == 0u ? 0x00400000u : b << 23);
}
#endif

// ---------------------------------------------------------------------------
// Norm over many tensors (k_clip.hip)
// ---------------------------------------------------------------------------
constexpr int kClipTensors = 150;      // tensors of a launch: 3000 bytes of arguments
constexpr int kClipChunk = 16384;      // elements of a workgroup at a time
constexpr uint32_t kClipBlocks = 2048; // workgroups of a launch, at most
constexpr uint32_t kClipSmall = 4;     // chunks that one workgroup takes, up to the factor

struct ClipTensor {
    void* g;
    int64_t n_bf16;   // elements, times two, plus one for bf16
};
struct ClipArgs {
    ClipTensor t[kClipTensors];
    uint32_t first[kClipTensors];  // a tensor's first chunk among the launch's
    int32_t count;
    uint32_t chunks;
};
// The sums of squares of a launch's tensors: *parts entries of `part`.
hipError_t launch_squares(const ClipArgs& a, double* part, int* parts, hipStream_t s);
// The norm of `scale` times the elements behind `parts` entries, and the factor for them, the
// product of two floats.
hipError_t launch_norm_factor(const double* part, int parts, double scale, double max_norm,
                              float* norm, float* factor, hipStream_t s);
// Both at once, of up to kClipSmall chunks.
hipError_t launch_norm_small(const ClipArgs& a, double scale, double max_norm, float* norm,
                             float* factor, hipStream_t s);
hipError_t launch_scale(const ClipArgs& a, const float* factor, hipStream_t s);

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
    const float* factor;  // two floats whose product is in place of grad_scale, or null
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
    bool vec_h;           // answers: h alone (vec: w)
    // log probabilities
    const uint8_t* w_scales;  // of a table in 8 bits, whose codes are w; or null
    int64_t ld_scales;
    const float* dlogp;       // backward, each or null
    const float* dentropy;
    float* entropy;           // forward: written, backward: read
    float* logp;
    int32_t top;              // classes to find, 0 .. kMostTop
    int32_t* ids;
    float* top_logp;
};
hipError_t launch_softmax_loss(const SoftmaxArgs& a, hipStream_t s);
hipError_t launch_softmax_grad(const SoftmaxArgs& a, hipStream_t s);

// ---------------------------------------------------------------------------
// Log probabilities (k_answer.hip)
// ---------------------------------------------------------------------------
constexpr int kMostTop = 64;

// How a call of n rows is laid out, from its sizes alone: `rows` rows and `piece`
// classes at a time.
struct AnswerPlan {
    SoftmaxPlan sm;
    int32_t few;                             // blocks of 16 rows, or 0: more than few
    bool thirds;                             // few fp32 rows in three bf16 parts
    int32_t group;                           // classes of a tile
    int32_t keep;                            // tiles that are looked at
    int64_t piece, rows;
    size_t part, best, lists, running, total;  // workspace offsets
};
AnswerPlan answer_plan(int64_t classes, int64_t n, int32_t dim, int32_t dtype, bool codes,
                       int32_t top);
hipError_t launch_log_probs(const SoftmaxArgs& a, hipStream_t s);
hipError_t launch_log_probs_grad(const SoftmaxArgs& a, hipStream_t s);

}  // namespace huge
