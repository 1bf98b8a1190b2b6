// Layer norm of rows and its backward pass.
//
// A group of TPR threads holds a row in registers, NV times VEC elements a
// thread: the mean, then the sum of squares about it, each one reduction over
// the group, so the variance loses nothing to a large mean and the row is read
// once.  TPR is the smallest power of two that covers the row at NV = 1, then NV
// grows; rows above 2048 elements take a whole workgroup.  The weight gradients
// are sums over all rows: a group adds its rows' terms in registers, a workgroup
// its groups', and a second kernel the workgroups' rows of `partial`, always in
// the same order.  Both kernels are bound by memory: a row is moved once in each
// direction.
#include "device.hpp"
#include "head.hpp"

namespace huge {

namespace {

template <int VEC>
struct Few {
    float v[VEC];
};

template <int VEC, typename E>
__device__ __forceinline__ Few<VEC> load_few(const E* __restrict__ row, int c) {
    Few<VEC> f;
    if constexpr (VEC == 4) {
        const float4 q = load_chunk(row, c);
        f.v[0] = q.x, f.v[1] = q.y, f.v[2] = q.z, f.v[3] = q.w;
    } else if constexpr (sizeof(E) == 4) {
        f.v[0] = row[c];
    } else {
        f.v[0] = __uint_as_float((uint32_t)row[c] << 16);
    }
    return f;
}

template <int VEC, typename E>
__device__ __forceinline__ void store_few(E* __restrict__ row, int c, const Few<VEC>& f) {
    if constexpr (VEC == 4) {
        store_chunk(row, c, make_float4(f.v[0], f.v[1], f.v[2], f.v[3]));
    } else if constexpr (sizeof(E) == 4) {
        row[c] = f.v[0];
    } else {
        row[c] = (bf16_t)float_to_bf16_bits(f.v[0]);
    }
}

// Sum over the TPR threads of a row.  Above a wave the four waves' sums meet in
// s_sum, whose two halves take turns so that one barrier a sum is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* s_sum, int& turn) {
    if constexpr (TPR <= 64) {
        return group_sum<TPR>(v);
    } else {
        v = group_sum<64>(v);
        float* s = s_sum + 4 * (turn++ & 1);
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        return (s[0] + s[1]) + (s[2] + s[3]);
    }
}

template <typename E, int TPR, int NV, int VEC>
__global__ __launch_bounds__(kBlock) void k_norm(NormArgs a) {
    __shared__ float s_sum[8];
    int turn = 0;
    constexpr int kRows = kBlock / TPR;
    const int t = threadIdx.x % TPR, D = a.dim, chunks = D / VEC;
    const E* x = static_cast<const E*>(a.x);
    E* y = static_cast<E*>(a.y);
    const float inv = 1.0f / (float)D;
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; r < a.n;
         r += (int64_t)gridDim.x * kRows) {
        Few<VEC> f[NV];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            f[i] = c < chunks ? load_few<VEC>(x + r * a.ld_x, c) : Few<VEC>{};
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum += f[i].v[e];
        }
        const float mean = row_sum<TPR>(sum, s_sum, turn) * inv;
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool in = t + TPR * i < chunks;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                f[i].v[e] -= mean;
                if (in) sq = fmaf(f[i].v[e], f[i].v[e], sq);
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(sq, s_sum, turn) * inv + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            if (c >= chunks) continue;
            const Few<VEC> g = load_few<VEC>(a.gamma, c), b = load_few<VEC>(a.beta, c);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[i].v[e] = fmaf(f[i].v[e] * rstd, g.v[e], b.v[e]);
            store_few<VEC>(y + r * a.ld_y, c, f[i]);
        }
        if (t == 0 && a.mean != nullptr) {
            a.mean[r] = mean;
            a.rstd[r] = rstd;
        }
    }
}

template <typename E, int TPR, int NV, int VEC>
__global__ __launch_bounds__(kBlock) void k_norm_backward(NormArgs a) {
    __shared__ float s_sum[8];
    int turn = 0;
    constexpr int kRows = kBlock / TPR;
    constexpr int kHeld = TPR < 64 ? TPR : 64;  // lanes of a wave that hold different columns
    const int t = threadIdx.x % TPR, D = a.dim, chunks = D / VEC;
    const E* x = static_cast<const E*>(a.x);
    const E* dy = static_cast<const E*>(a.dy);
    E* dx = static_cast<E*>(a.y);
    const float inv = 1.0f / (float)D;
    Few<VEC> g[NV], dg[NV], db[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = t + TPR * i;
        g[i] = c < chunks ? load_few<VEC>(a.gamma, c) : Few<VEC>{};
        dg[i] = db[i] = Few<VEC>{};
    }
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; r < a.n;
         r += (int64_t)gridDim.x * kRows) {
        const float mean = a.mean[r], rstd = a.rstd[r];
        Few<VEC> xh[NV], d[NV];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            const bool in = c < chunks;
            xh[i] = in ? load_few<VEC>(x + r * a.ld_x, c) : Few<VEC>{};
            d[i] = in ? load_few<VEC>(dy + r * a.ld_dy, c) : Few<VEC>{};
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool in = t + TPR * i < chunks;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                xh[i].v[e] = in ? (xh[i].v[e] - mean) * rstd : 0.f;
                dg[i].v[e] = fmaf(d[i].v[e], xh[i].v[e], dg[i].v[e]);
                db[i].v[e] += d[i].v[e];
                d[i].v[e] *= g[i].v[e];
                s1 += d[i].v[e];
                s2 = fmaf(d[i].v[e], xh[i].v[e], s2);
            }
        }
        if (dx == nullptr) continue;
        s1 = row_sum<TPR>(s1, s_sum, turn) * inv;
        s2 = row_sum<TPR>(s2, s_sum, turn) * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            if (c >= chunks) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                d[i].v[e] = rstd * (d[i].v[e] - s1 - xh[i].v[e] * s2);
            store_few<VEC>(dx + r * a.ld_y, c, d[i]);
        }
    }
    if (a.partial == nullptr) return;
    // the groups of a wave, then the waves
    __shared__ float s_part[TPR <= 64 ? 4 * kHeld * NV * VEC : 1];
    float* out = a.partial + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        Few<VEC>* p = which == 0 ? dg : db;
        if constexpr (TPR <= 64) {
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float v = p[i].v[e];
#pragma unroll
                    for (int off = TPR; off < 64; off <<= 1) v += __shfl_xor(v, off);
                    if (lane < kHeld) s_part[((wave * NV + i) * VEC + e) * kHeld + lane] = v;
                }
            __syncthreads();
            for (int j = threadIdx.x; j < D; j += kBlock) {
                const int c = j / VEC, at = ((c / TPR) * VEC + j % VEC) * kHeld + c % TPR;
                constexpr int kWave = NV * VEC * kHeld;
                out[(int64_t)which * D + j] = (s_part[at] + s_part[kWave + at]) +
                                              (s_part[2 * kWave + at] + s_part[3 * kWave + at]);
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = t + TPR * i;
                if (c >= chunks) continue;
#pragma unroll
                for (int e = 0; e < VEC; ++e) out[(int64_t)which * D + c * VEC + e] = p[i].v[e];
            }
        }
    }
}

// Column sums of `partial`: a workgroup takes 16 columns, 16 threads each.
__global__ __launch_bounds__(kBlock) void k_norm_reduce(const float* __restrict__ partial,
                                                        int blocks, int dim,
                                                        float* __restrict__ dgamma,
                                                        float* __restrict__ dbeta) {
    __shared__ float s[16][17];
    const int col = blockIdx.x * 16 + (threadIdx.x & 15), lane = threadIdx.x >> 4;
    float v = 0.f;
    if (col < 2 * dim) {
#pragma unroll 8
        for (int b = lane; b < blocks; b += 16) v += partial[(int64_t)b * 2 * dim + col];
    }
    s[lane][threadIdx.x & 15] = v;
    __syncthreads();
    if (lane == 0 && col < 2 * dim) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) sum += s[k][threadIdx.x & 15];
        if (col < dim) dgamma[col] = sum;
        else dbeta[col - dim] = sum;
    }
}

struct NormShape {
    int tpr, nv;
};

// Threads of a row and vectors a thread, of `units` vectors (or elements).
inline NormShape norm_shape(int units, bool vec) {
    const int one = vec ? 8 : 64;  // fewest threads of a row
    int tpr = one;
    while (tpr < 64 && tpr < units) tpr <<= 1;
    int nv = 1;
    const int most = vec ? 8 : 32;
    while (tpr * nv < units && nv < most) nv <<= 1;
    return tpr * nv < units ? NormShape{kBlock, most} : NormShape{tpr, nv};
}

template <typename E, int TPR, int NV, int VEC>
void norm_one(const NormArgs& a, bool backward, hipStream_t s) {
    const int64_t rows = kBlock / TPR, need = (a.n + rows - 1) / rows;
    if (!backward) {
        const int64_t grid = need < 65536 ? need : 65536;
        k_norm<E, TPR, NV, VEC><<<dim3((uint32_t)grid), kBlock, 0, s>>>(a);
    } else {
        k_norm_backward<E, TPR, NV, VEC>
            <<<dim3((uint32_t)norm_blocks(a.n, a.dim)), kBlock, 0, s>>>(a);
    }
}

template <typename E>
hipError_t norm_dispatch(const NormArgs& a, bool backward, hipStream_t s) {
    const NormShape p = norm_shape(a.vec ? a.dim / 4 : a.dim, a.vec);
#define HUGE_NORM_CASE(T, N, V) \
    case (T) * 64 + (N):        \
        norm_one<E, T, N, V>(a, backward, s); \
        return hipGetLastError();
    if (a.vec) {
        switch (p.tpr * 64 + p.nv) {
            HUGE_NORM_CASE(8, 1, 4)
            HUGE_NORM_CASE(16, 1, 4)
            HUGE_NORM_CASE(32, 1, 4)
            HUGE_NORM_CASE(64, 1, 4)
            HUGE_NORM_CASE(64, 2, 4)
            HUGE_NORM_CASE(64, 4, 4)
            HUGE_NORM_CASE(64, 8, 4)
            HUGE_NORM_CASE(256, 8, 4)
        }
    } else {
        switch (p.tpr * 64 + p.nv) {
            HUGE_NORM_CASE(64, 1, 1)
            HUGE_NORM_CASE(64, 2, 1)
            HUGE_NORM_CASE(64, 4, 1)
            HUGE_NORM_CASE(64, 8, 1)
            HUGE_NORM_CASE(64, 16, 1)
            HUGE_NORM_CASE(64, 32, 1)
            HUGE_NORM_CASE(256, 32, 1)
        }
    }
#undef HUGE_NORM_CASE
    return hipErrorInvalidValue;
}

}  // namespace

// A workgroup sums at least 16 rows a group, so that small calls have few rows of
// partial sums.
int norm_blocks(int64_t n, int32_t dim) {
    const int64_t rows = dim > 2048 ? 1 : 4;
    const int64_t b = (n + 16 * rows - 1) / (16 * rows);
    return (int)(b < kNormBlocks ? b : kNormBlocks);
}

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
    return a.dtype == kDtypeBf16 ? norm_dispatch<bf16_t>(a, false, s)
                                 : norm_dispatch<float>(a, false, s);
}

hipError_t launch_norm_backward(const NormArgs& a, float* dgamma, float* dbeta, hipStream_t s) {
    if (a.n > 0) {
        const hipError_t e = a.dtype == kDtypeBf16 ? norm_dispatch<bf16_t>(a, true, s)
                                                   : norm_dispatch<float>(a, true, s);
        if (e != hipSuccess) return e;
    }
    if (dgamma == nullptr) return hipSuccess;
    k_norm_reduce<<<dim3((uint32_t)((2 * a.dim + 15) / 16)), kBlock, 0, s>>>(
        a.partial, norm_blocks(a.n, a.dim), a.dim, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace huge
