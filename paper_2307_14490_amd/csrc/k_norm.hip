// Layer norm of rows and its backward pass.
//
// A group of TPR threads holds a row in registers, NV times four elements a
// thread: the mean, then the sum of squares about it, each one reduction over
// the group, so the variance loses nothing to a large mean and the row is read
// once.  TPR is the smallest power of two that covers the row at NV = 1, then NV
// grows; rows above 1024 elements take a whole workgroup.  The weight gradients
// are sums over all rows: a group adds its rows' terms in registers, a workgroup
// its groups', and a second kernel the workgroups' rows of `partial`, always in
// the same order.  Both kernels are bound by memory: a row is moved once in each
// direction.
//
// Measured, bytes that have to be moved over time (a copy reaches 4.8 TB/s): 262144
// x 256 fp32 95 us forward (5.6 TB/s), 157 us backward (5.1) and 5 us for the second
// kernel; 65536 x 128 bf16, which stays in the caches, 12, 13 and 5 us.  Rows that
// are not whole aligned fours: 60417 x 761 both ways 188 us in fp32 (4.9 TB/s, as
// with 760 columns), 154 us in bf16 (3.0; 760 columns: 101 us), where an 8-byte
// access at an odd address is taken apart; one element a thread took 279 us.  Rows
// above 1024 columns by a wave alone would hold 8 chunks of three arrays a thread,
// two waves per SIMD: 60417 x 2048 bf16 387 us against 286 by a workgroup.
#include "rows.hpp"

namespace huge {

namespace {

template <typename E, int TPR, int NV, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_norm(NormArgs a) {
    __shared__ float s_sum[8];
    int turn = 0;
    constexpr int kRows = kBlock / TPR;
    const int t = threadIdx.x % TPR, D = a.dim, chunks = (D + 3) / 4;
    const E* x = static_cast<const E*>(a.x);
    E* y = static_cast<E*>(a.y);
    const float inv = 1.0f / (float)D;
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; r < a.n;
         r += (int64_t)gridDim.x * kRows) {
        Few f[NV];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            f[i] = c < chunks ? load_few<WHOLE>(x + r * a.ld_x, c, D) : Few{};
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += f[i].v[e];
        }
        const float mean = row_sum<TPR>(sum, s_sum, turn) * inv;
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[i].v[e] -= mean;
                if (inside<WHOLE>(c, e, D)) sq = fmaf(f[i].v[e], f[i].v[e], sq);
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(sq, s_sum, turn) * inv + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            if (c >= chunks) continue;
            const Few g = load_few<WHOLE>(a.gamma, c, D), b = load_few<WHOLE>(a.beta, c, D);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[i].v[e] = fmaf(f[i].v[e] * rstd, g.v[e], b.v[e]);
            store_few<WHOLE>(y + r * a.ld_y, c, D, f[i]);
        }
        if (t == 0 && a.mean != nullptr) {
            a.mean[r] = mean;
            a.rstd[r] = rstd;
        }
    }
}

template <typename E, int TPR, int NV, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_norm_backward(NormArgs a) {
    __shared__ float s_sum[8];
    int turn = 0;
    constexpr int kRows = kBlock / TPR;
    constexpr int kHeld = TPR < 64 ? TPR : 64;  // lanes of a wave that hold different columns
    const int t = threadIdx.x % TPR, D = a.dim, chunks = (D + 3) / 4;
    const E* x = static_cast<const E*>(a.x);
    const E* dy = static_cast<const E*>(a.dy);
    E* dx = static_cast<E*>(a.y);
    const float inv = 1.0f / (float)D;
    Few g[NV], dg[NV], db[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = t + TPR * i;
        g[i] = c < chunks ? load_few<WHOLE>(a.gamma, c, D) : Few{};
        dg[i] = db[i] = Few{};
    }
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; r < a.n;
         r += (int64_t)gridDim.x * kRows) {
        const float mean = a.mean[r], rstd = a.rstd[r];
        Few xh[NV], d[NV];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            const bool in = c < chunks;
            xh[i] = in ? load_few<WHOLE>(x + r * a.ld_x, c, D) : Few{};
            d[i] = in ? load_few<WHOLE>(dy + r * a.ld_dy, c, D) : Few{};
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                xh[i].v[e] = inside<WHOLE>(c, e, D) ? (xh[i].v[e] - mean) * rstd : 0.f;
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
            for (int e = 0; e < 4; ++e)
                d[i].v[e] = rstd * (d[i].v[e] - s1 - xh[i].v[e] * s2);
            store_few<WHOLE>(dx + r * a.ld_y, c, D, d[i]);
        }
    }
    if (a.partial == nullptr) return;
    // the groups of a wave, then the waves
    __shared__ float s_part[TPR <= 64 ? 4 * kHeld * NV * 4 : 1];
    float* out = a.partial + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        Few* p = which == 0 ? dg : db;
        if constexpr (TPR <= 64) {
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v = p[i].v[e];
#pragma unroll
                    for (int off = TPR; off < 64; off <<= 1) v += __shfl_xor(v, off);
                    if (lane < kHeld) s_part[((wave * NV + i) * 4 + e) * kHeld + lane] = v;
                }
            __syncthreads();
            for (int j = threadIdx.x; j < D; j += kBlock) {
                const int c = j / 4, at = ((c / TPR) * 4 + j % 4) * kHeld + c % TPR;
                constexpr int kWave = NV * 4 * kHeld;
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
                for (int e = 0; e < 4; ++e)
                    if (inside<WHOLE>(c, e, D)) out[(int64_t)which * D + c * 4 + e] = p[i].v[e];
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

template <typename E, int TPR, int NV, bool WHOLE>
void norm_one(const NormArgs& a, bool backward, hipStream_t s) {
    const int64_t rows = kBlock / TPR, need = (a.n + rows - 1) / rows;
    if (!backward) {
        const int64_t grid = need < 65536 ? need : 65536;
        k_norm<E, TPR, NV, WHOLE><<<dim3((uint32_t)grid), kBlock, 0, s>>>(a);
    } else {
        k_norm_backward<E, TPR, NV, WHOLE>
            <<<dim3((uint32_t)norm_blocks(a.n, a.dim)), kBlock, 0, s>>>(a);
    }
}

template <typename E>
hipError_t norm_dispatch(const NormArgs& a, bool backward, hipStream_t s) {
    const NormShape p = norm_shape((a.dim + 3) / 4);
#define HUGE_NORM_CASE(T, N)                           \
    case (T) * 64 + (N):                               \
        if (a.vec) norm_one<E, T, N, true>(a, backward, s); \
        else norm_one<E, T, N, false>(a, backward, s); \
        return hipGetLastError();
    switch (p.tpr * 64 + p.nv) {
        HUGE_NORM_CASE(8, 1)
        HUGE_NORM_CASE(16, 1)
        HUGE_NORM_CASE(32, 1)
        HUGE_NORM_CASE(64, 1)
        HUGE_NORM_CASE(64, 2)
        HUGE_NORM_CASE(64, 4)
        HUGE_NORM_CASE(256, 2)
        HUGE_NORM_CASE(256, 4)
        HUGE_NORM_CASE(256, 8)
    }
#undef HUGE_NORM_CASE
    return hipErrorInvalidValue;
}

}  // namespace

// A workgroup sums at least 16 rows a group, so that small calls have few rows of
// partial sums.
int norm_blocks(int64_t n, int32_t dim) {
    const int64_t rows = dim > 1024 ? 1 : 4;
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
