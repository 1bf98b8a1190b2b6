// Rows held in registers by a group of threads, four elements at a time: what the
// kernels that normalise rows share (k_norm.hip, k_rms.hip).
#pragma once

#include "device.hpp"
#include "head.hpp"

namespace huge {

namespace {

// Four elements of a row.
struct Few {
    float v[4];
};

typedef float raw_f4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t raw_h4 __attribute__((ext_vector_type(4), aligned(2)));

// Chunk c of a row of D elements.  WHOLE: D is a multiple of four and the rows lie
// on whole chunks.  Otherwise the load needs no more than the element's alignment,
// and the row's last chunk is read one by one, with zeros past the end.
template <bool WHOLE, typename E>
__device__ __forceinline__ Few load_few(const E* __restrict__ row, int c, int D) {
    Few f{};
    if constexpr (WHOLE) {
        const float4 q = load_chunk(row, c);
        f.v[0] = q.x, f.v[1] = q.y, f.v[2] = q.z, f.v[3] = q.w;
    } else if (4 * c + 4 <= D) {
        if constexpr (sizeof(E) == 4) {
            const raw_f4 q = *reinterpret_cast<const raw_f4*>(row + 4 * c);
#pragma unroll
            for (int e = 0; e < 4; ++e) f.v[e] = q[e];
        } else {
            const raw_h4 q = *reinterpret_cast<const raw_h4*>(row + 4 * c);
#pragma unroll
            for (int e = 0; e < 4; ++e) f.v[e] = __uint_as_float((uint32_t)q[e] << 16);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            if (4 * c + e >= D) continue;
            if constexpr (sizeof(E) == 4) f.v[e] = row[4 * c + e];
            else f.v[e] = __uint_as_float((uint32_t)row[4 * c + e] << 16);
        }
    }
    return f;
}

template <bool WHOLE, typename E>
__device__ __forceinline__ void store_few(E* __restrict__ row, int c, int D, const Few& f) {
    if constexpr (WHOLE) {
        store_chunk(row, c, make_float4(f.v[0], f.v[1], f.v[2], f.v[3]));
    } else if (4 * c + 4 <= D) {
        if constexpr (sizeof(E) == 4) {
            *reinterpret_cast<raw_f4*>(row + 4 * c) = raw_f4{f.v[0], f.v[1], f.v[2], f.v[3]};
        } else {
            raw_h4 q;
#pragma unroll
            for (int e = 0; e < 4; ++e) q[e] = (bf16_t)float_to_bf16_bits(f.v[e]);
            *reinterpret_cast<raw_h4*>(row + 4 * c) = q;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            if (4 * c + e >= D) continue;
            if constexpr (sizeof(E) == 4) row[4 * c + e] = f.v[e];
            else row[4 * c + e] = (bf16_t)float_to_bf16_bits(f.v[e]);
        }
    }
}

// Whether element e of chunk c is one of the row's.
template <bool WHOLE>
__device__ __forceinline__ bool inside(int c, int e, int D) {
    return WHOLE ? 4 * c < D : 4 * c + e < D;
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

struct NormShape {
    int tpr, nv;
};

// Threads of a row and chunks a thread, of `chunks` chunks.
inline NormShape norm_shape(int chunks) {
    int tpr = 8, nv = 1;
    while (tpr < 64 && tpr < chunks) tpr <<= 1;
    while (tpr * nv < chunks && nv < 4) nv <<= 1;
    if (tpr * nv >= chunks) return {tpr, nv};
    for (nv = 2; kBlock * nv < chunks; nv <<= 1) {}
    return {kBlock, nv};
}

}  // namespace

}  // namespace huge
