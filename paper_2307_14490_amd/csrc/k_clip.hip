// The 2-norm over all elements of many tensors, and scaling by a factor that it gives.
//
// A workgroup takes chunks of 16384 elements of the launch's tensors (their table is in
// the kernel's arguments) in turn and adds their squares in fp64, in which a square
// of either type is exact and cannot overflow or vanish; its sum is one entry of
// `part`.  A second kernel adds the entries, always in the same order, and writes the
// norm and the factor, which stay on the device: what applies it (AdamW's step, or
// k_scale in place) reads it there.  Bound by memory, each gradient being read once: 129e6
// fp32 elements 118 to 132 us (3.9 to 4.4 TB/s; a read reaches 4.0), 40e6 bf16 ones in
// 400 tensors 24 us in three launches of up to 150 tensors.  In place 129e6 fp32 elements take 159 us
// more (6.5 TB/s), 285 in all.
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

// A chunk's elements.
struct Chunk {
    void* p;
    int64_t left;  // elements of the tensor from p on
    bool bf16;
};
// The tensor that holds a chunk is the last whose first is not above it.
__device__ __forceinline__ Chunk chunk_of(const ClipArgs& a, uint32_t chunk) {
    int lo = 0, hi = a.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    const ClipTensor& t = a.t[lo];
    const bool bf16 = t.n_bf16 & 1;
    const int64_t at = (int64_t)(chunk - a.first[lo]) * kClipChunk;
    return {static_cast<uint8_t*>(t.g) + at * (bf16 ? 2 : 4), (t.n_bf16 >> 1) - at, bf16};
}

// Calls body(pointer) for a thread's 16-byte pieces of a chunk, and one(pointer) for the
// elements before the first and behind the last aligned one.
// kBlock threads share a chunk.
template <typename E, typename Body, typename One>
__device__ __forceinline__ void each(E* p, int64_t left, Body body, One one) {
    constexpr int W = kWide<E>;
    const int tid = threadIdx.x % kBlock;
    const int n = (int)(left < kClipChunk ? left : kClipChunk);
    const int off = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(E));
    const int skip = off == 0 ? 0 : W - off < n ? W - off : n;
    const int wide = (n - skip) / W;
    if (wide == kClipChunk / W) {
#pragma unroll 8
        for (int k = 0; k < kClipChunk / W; k += kBlock) body(p + skip + (k + tid) * W);
    } else {
#pragma unroll 4
        for (int k = tid; k < wide; k += kBlock) body(p + skip + k * W);
    }
    if (tid < skip) one(p + tid);
    const int end = skip + wide * W;
    if (tid < n - end) one(p + end + tid);
}

// Sum of the squares of a thread's elements of a chunk.
template <typename E>
__device__ __forceinline__ double squares(E* p, int64_t left) {
    double s[2] = {0.0, 0.0};
    each<E>(
        p, left,
        [&](const E* at) {
            const Sixteen<E> q = load_sixteen(at);
#pragma unroll
            for (int e = 0; e < kWide<E>; ++e) {
                const double x = (double)q.v[e];
                s[e & 1] = fma(x, x, s[e & 1]);
            }
        },
        [&](const E* at) {
            const double x = (double)load_one(at);
            s[0] = fma(x, x, s[0]);
        });
    return s[0] + s[1];
}
__device__ __forceinline__ double squares(const Chunk& c) {
    return c.bf16 ? squares(static_cast<bf16_t*>(c.p), c.left)
                  : squares(static_cast<float*>(c.p), c.left);
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
    // from the last chunk on: the step that follows starts at the first, whose elements are then
    // the last that were read (129e6 fp32 elements and AdamW's step: 704 -> 694 us)
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x)
        v += squares(chunk_of(a, a.chunks - 1 - c));
    v = block_sum<kBlock>(v, s);
    if (threadIdx.x == 0) part[blockIdx.x] = v;
}

// The norm of `scale` times the elements from the sum of their squares, and the factor
// for them: scale, or less so that the norm is max_norm.  NaN where the norm is not finite.  It is
// the product of two floats, one after the other: below 2^-126 (a norm of 1e38 brought to 1) one
// alone would lose digits or be 0.
__device__ __forceinline__ void write_factor(double square, double scale, double max_norm,
                                             float* norm, float* factor) {
    const double r = fabs(scale) * sqrt(square);
    if (norm != nullptr) *norm = (float)r;
    const double f = r > max_norm ? scale * (max_norm / r) : scale;
    const bool small = fabs(f) < 0x1p-126;
    factor[0] = !(r < INFINITY) ? NAN : (float)(small ? f * 0x1p126 : f);
    factor[1] = small ? 0x1p-126f : 1.0f;
}

__global__ __launch_bounds__(1024) void k_norm_factor(const double* __restrict__ part, int n,
                                                      double scale, double max_norm,
                                                      float* __restrict__ norm,
                                                      float* __restrict__ factor) {
    __shared__ double s[16];
    double v = 0.0;
#pragma unroll 4
    for (int k = threadIdx.x; k < n; k += 1024) v += part[k];
    v = block_sum<1024>(v, s);
    if (threadIdx.x == 0) write_factor(v, scale, max_norm, norm, factor);
}

// A few chunks: by one workgroup at once, in one launch.
__global__ __launch_bounds__(1024) void k_norm_small(ClipArgs a, double scale, double max_norm,
                                                     float* __restrict__ norm,
                                                     float* __restrict__ factor) {
    __shared__ double s[16];
    double v = 0.0;
    static_assert(kClipSmall * kBlock <= 1024, "a chunk has kBlock threads");
    const uint32_t c = threadIdx.x / kBlock;
    if (c < a.chunks) v = squares(chunk_of(a, c));
    v = block_sum<1024>(v, s);
    if (threadIdx.x == 0) write_factor(v, scale, max_norm, norm, factor);
}

template <typename E>
__device__ __forceinline__ void scale_chunk(E* p, int64_t left, float f, float f2) {
    each<E>(
        p, left,
        [&](E* at) {
            const Sixteen<E> q = load_sixteen(at);
            if constexpr (sizeof(E) == 4) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = q.v[e] * f * f2;
                *reinterpret_cast<f32x4*>(at) = v;
            } else {
                f32x8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = q.v[e] * f * f2;
                *reinterpret_cast<bf16x8*>(at) = __builtin_convertvector(v, bf16x8);
            }
        },
        [&](E* at) {
            const float v = load_one(at) * f * f2;
            if constexpr (sizeof(E) == 4) *at = v;
            else *at = (bf16_t)float_to_bf16_bits(v);
        });
}

// Nothing is read or written where the factor is 1, or no number.
__global__ __launch_bounds__(kBlock) void k_scale(ClipArgs a, const float* __restrict__ factor) {
    const float f = factor[0], f2 = factor[1];
    if ((f == 1.0f && f2 == 1.0f) || f != f) return;
    for (uint32_t k = blockIdx.x; k < a.chunks; k += gridDim.x) {
        const Chunk c = chunk_of(a, k);
        if (c.bf16) scale_chunk(static_cast<bf16_t*>(c.p), c.left, f, f2);
        else scale_chunk(static_cast<float*>(c.p), c.left, f, f2);
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

hipError_t launch_norm_small(const ClipArgs& a, double scale, double max_norm, float* norm,
                             float* factor, hipStream_t s) {
    k_norm_small<<<1, 1024, 0, s>>>(a, scale, max_norm, norm, factor);
    return hipGetLastError();
}

hipError_t launch_scale(const ClipArgs& a, const float* factor, hipStream_t s) {
    k_scale<<<dim3(clip_blocks(a)), kBlock, 0, s>>>(a, factor);
    return hipGetLastError();
}

}  // namespace huge
