// The 2-norm over all elements of many tensors, and scaling by a factor that it gives.
//
// A workgroup takes chunks of 16384 elements of the launch's tensors (their table is in
// the kernel's arguments) in turn and adds their squares in fp64, in which a square
// of either type is exact and cannot overflow or vanish; its sum is one entry of
// `part`.  A second kernel adds the entries, always in the same order, and writes the
// norm and the factor, which stay on the device: what applies it (AdamW's step, or
// k_scale in place) reads it there.  Bound by memory: each gradient is read once.
#include "device.hpp"
#include "head.hpp"

namespace huge {

namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename E>
constexpr int kWide = 16 / sizeof(E);  // elements of 16 bytes

template <typename E>
struct Sixteen {
    float v[kWide<E>];
};

template <typename E>
__device__ __forceinline__ Sixteen<E> load_sixteen(const E* p) {
    Sixteen<E> r;
    if constexpr (sizeof(E) == 4) {
        const f32x4 q = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) r.v[e] = q[e];
    } else {
        const u16x8 q = *reinterpret_cast<const u16x8*>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = __uint_as_float((uint32_t)q[e] << 16);
    }
    return r;
}

template <typename E>
__device__ __forceinline__ float load_one(const E* p) {
    if constexpr (sizeof(E) == 4) return *p;
    else return __uint_as_float((uint32_t)*p << 16);
}

// The tensor whose chunks hold `chunk`: the last whose first is not above it.
__device__ __forceinline__ const ClipTensor& tensor_of(const ClipArgs& a, uint32_t chunk) {
    int k = 0;
    for (int j = 1; j < a.count; ++j)
        if (a.t[j].first <= chunk) k = j;
    return a.t[k];
}

// Sum of the squares of a thread's elements of a chunk of n.
template <typename E>
__device__ __forceinline__ double squares(const E* p, int64_t n, bool vec) {
    constexpr int W = kWide<E>, kStep = kBlock * W;
    double s[2] = {0.0, 0.0};
    if (vec && n >= kClipChunk) {
#pragma unroll 4
        for (int k = 0; k < kClipChunk; k += kStep) {
            const Sixteen<E> q = load_sixteen(p + k + threadIdx.x * W);
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const double x = (double)q.v[e];
                s[e & 1] = fma(x, x, s[e & 1]);
            }
        }
    } else {
        const int m = (int)(n < kClipChunk ? n : kClipChunk);
#pragma unroll 4
        for (int k = threadIdx.x; k < m; k += kBlock) {
            const double x = (double)load_one(p + k);
            s[0] = fma(x, x, s[0]);
        }
    }
    return s[0] + s[1];
}

// Sum over a workgroup, in thread 0.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* s) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_down(v, off);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int k = 1; k < THREADS / 64; ++k) v += s[k];
    return v;
}

__global__ __launch_bounds__(kBlock) void k_squares(ClipArgs a, double* __restrict__ part) {
    __shared__ double s[kBlock / 64];
    double v = 0.0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipTensor& t = tensor_of(a, c);
        const int64_t at = (int64_t)(c - t.first) * kClipChunk;
        if (t.dtype == kDtypeBf16)
            v += squares(static_cast<const bf16_t*>(t.g) + at, t.n - at, t.vec);
        else
            v += squares(static_cast<const float*>(t.g) + at, t.n - at, t.vec);
    }
    v = block_sum<kBlock>(v, s);
    if (threadIdx.x == 0) part[blockIdx.x] = v;
}

// The norm of `scale` times the elements, and the factor for them: scale, or less so that
// the norm is max_norm.  NaN where the norm is not finite.
__global__ __launch_bounds__(1024) void k_norm_factor(const double* __restrict__ part, int n,
                                                      double scale, double max_norm,
                                                      float* __restrict__ norm,
                                                      float* __restrict__ factor) {
    __shared__ double s[16];
    double v = 0.0;
    for (int k = threadIdx.x; k < n; k += 1024) v += part[k];
    v = block_sum<1024>(v, s);
    if (threadIdx.x != 0) return;
    const double r = fabs(scale) * sqrt(v);
    if (norm != nullptr) *norm = (float)r;
    if (factor != nullptr)
        *factor = !(r < INFINITY) ? NAN : (float)(r > max_norm ? scale * (max_norm / r) : scale);
}

template <typename E>
__device__ __forceinline__ void scale_chunk(E* p, int64_t n, bool vec, float f) {
    constexpr int W = kWide<E>, kStep = kBlock * W;
    if (vec && n >= kClipChunk) {
#pragma unroll 4
        for (int k = 0; k < kClipChunk; k += kStep) {
            E* at = p + k + threadIdx.x * W;
            const Sixteen<E> q = load_sixteen(at);
            if constexpr (sizeof(E) == 4) {
                *reinterpret_cast<f32x4*>(at) = f32x4{q.v[0] * f, q.v[1] * f, q.v[2] * f, q.v[3] * f};
            } else {
                f32x8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = q.v[e] * f;
                *reinterpret_cast<bf16x8*>(at) = __builtin_convertvector(v, bf16x8);
            }
        }
    } else {
        const int m = (int)(n < kClipChunk ? n : kClipChunk);
        for (int k = threadIdx.x; k < m; k += kBlock) {
            const float v = load_one(p + k) * f;
            if constexpr (sizeof(E) == 4) p[k] = v;
            else p[k] = (bf16_t)float_to_bf16_bits(v);
        }
    }
}

// Nothing is read or written where the factor is 1, or no number.
__global__ __launch_bounds__(kBlock) void k_scale(ClipArgs a, const float* __restrict__ factor) {
    const float f = *factor;
    if (f == 1.0f || f != f) return;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipTensor& t = tensor_of(a, c);
        const int64_t at = (int64_t)(c - t.first) * kClipChunk;
        if (t.dtype == kDtypeBf16)
            scale_chunk(static_cast<bf16_t*>(t.g) + at, t.n - at, t.vec, f);
        else
            scale_chunk(static_cast<float*>(t.g) + at, t.n - at, t.vec, f);
    }
}

uint32_t clip_blocks(const ClipArgs& a) { return a.chunks < kClipBlocks ? a.chunks : kClipBlocks; }

}  // namespace

hipError_t launch_squares(const ClipArgs& a, double* part, int* parts, hipStream_t s) {
    *parts = (int)clip_blocks(a);
    k_squares<<<dim3(clip_blocks(a)), kBlock, 0, s>>>(a, part);
    return hipGetLastError();
}

hipError_t launch_norm_factor(const double* part, int parts, double scale, double max_norm,
                              float* norm, float* factor, hipStream_t s) {
    k_norm_factor<<<1, 1024, 0, s>>>(part, parts, scale, max_norm, norm, factor);
    return hipGetLastError();
}

hipError_t launch_scale(const ClipArgs& a, const float* factor, hipStream_t s) {
    k_scale<<<dim3(clip_blocks(a)), kBlock, 0, s>>>(a, factor);
    return hipGetLastError();
}

}  // namespace huge
