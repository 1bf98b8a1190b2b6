// AdamW over many tensors, with moments as floats or in 8 bits.
//
// One pass: an element's parameter, gradient and moments are read, updated in
// registers and written.  A workgroup takes a chunk of kAdamChunk elements of one
// tensor, found in the launch's table (in the kernel's arguments); a wave takes
// 256 elements at a time, four a lane, which is one block of an 8-bit state: its
// scales are a maximum over the wave's registers.  Bound by memory.
//
// Every product and sum is rounded by itself (no contraction), so that a moment
// in 8 bits takes the same code wherever the same formula is computed in fp32: a
// value one unit away from where a code changes would otherwise move by a code,
// which is thousands of units.
#include <float.h>

#include "device.hpp"
#include "head.hpp"

#pragma clang fp contract(off)

namespace huge {

namespace {

constexpr float kInv127 = 1.0f / 127.0f;
constexpr float kInv255 = 1.0f / 255.0f;

template <typename E>
__device__ __forceinline__ void load4(const E* __restrict__ p, int64_t i, int64_t n, bool vec,
                                      float* v) {
    if (vec && i + 4 <= n) {
        const float4 q = load_chunk(p + i, 0);
        v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = 0.f;
        if (i + e < n) {
            if constexpr (sizeof(E) == 4) v[e] = p[i + e];
            else v[e] = __uint_as_float((uint32_t)p[i + e] << 16);
        }
    }
}

template <typename E>
__device__ __forceinline__ void store4(E* __restrict__ p, int64_t i, int64_t n, bool vec,
                                       const float* v) {
    if (vec && i + 4 <= n) {
        store_chunk(p + i, 0, make_float4(v[0], v[1], v[2], v[3]));
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i + e < n) {
            if constexpr (sizeof(E) == 4) p[i + e] = v[e];
            else p[i + e] = (bf16_t)float_to_bf16_bits(v[e]);
        }
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

// The moments of four elements at i (a multiple of 4) of a tensor of n.  `b`: the
// block of 256 that holds them.
template <bool Q8>
struct Moments;

template <>
struct Moments<false> {
    static __device__ __forceinline__ void load(const uint8_t* state, int64_t n, int64_t i,
                                                float* m, float* v) {
        // padded to whole blocks: always four at a time
        const float* sm = reinterpret_cast<const float*>(state);
        load4(sm, i, i + 4, true, m);
        load4(sm + adam_padded(n), i, i + 4, true, v);
    }
    static __device__ __forceinline__ void store(uint8_t* state, int64_t n, int64_t i,
                                                 const float* m, const float* v, const float*) {
        float* sm = reinterpret_cast<float*>(state);
        store4(sm, i, i + 4, true, m);
        store4(sm + adam_padded(n), i, i + 4, true, v);
    }
};

template <>
struct Moments<true> {
    static __device__ __forceinline__ float2* scales(uint8_t* state, int64_t n, int64_t i) {
        return reinterpret_cast<float2*>(state + 2 * adam_padded(n)) + i / kAdamBlock;
    }
    static __device__ __forceinline__ void load(const uint8_t* state, int64_t n, int64_t i,
                                                float* m, float* v) {
        const uint32_t q = *reinterpret_cast<const uint32_t*>(state + i);
        const uint32_t u = *reinterpret_cast<const uint32_t*>(state + adam_padded(n) + i);
        const float2 s = *scales(const_cast<uint8_t*>(state), n, i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float k = (float)(int8_t)(q >> (8 * e));
            const float a = fabsf(k) * kInv127;
            m[e] = copysignf(s.x * (a * a), k);
            const float c = (float)((u >> (8 * e)) & 0xFFu) * kInv255;
            const float r = s.y * (c * c);
            v[e] = r * r;
        }
    }
    // r: sqrt(v), 0 past the end of the tensor (as m is).  Every lane of the wave
    // takes part: its 256 elements are one block.
    static __device__ __forceinline__ void store(uint8_t* state, int64_t n, int64_t i,
                                                 const float* m, const float*, const float* r) {
        float s = fmaxf(fmaxf(fabsf(m[0]), fabsf(m[1])), fmaxf(fabsf(m[2]), fabsf(m[3])));
        float t = fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3]));
        s = wave_max(s);
        t = wave_max(t);
        // the reciprocal of a subnormal scale is kept finite, so that 0 keeps its code
        const float is = s > 0.f ? fminf(1.0f / s, FLT_MAX) : 0.f;
        const float it = t > 0.f ? 1.0f / t : 0.f;
        uint32_t q = 0, u = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = fminf(rintf(sqrtf(fabsf(m[e]) * is) * 127.0f), 127.0f);
            float c = fminf(rintf(sqrtf(r[e] * it) * 255.0f), 255.0f);
            if (r[e] > 0.f) c = fmaxf(c, 1.0f);
            const int k = m[e] < 0.f ? -(int)a : (int)a;
            q |= (uint32_t)(k & 0xFF) << (8 * e);
            u |= (uint32_t)c << (8 * e);
        }
        if (i >= adam_padded(n)) return;
        *reinterpret_cast<uint32_t*>(state + i) = q;
        *reinterpret_cast<uint32_t*>(state + adam_padded(n) + i) = u;
        if ((threadIdx.x & 63) == 0) *scales(state, n, i) = make_float2(s, t);
    }
};

// The tensor whose chunks hold this workgroup's: the last whose first is not
// above it.  Tensors without elements have no chunk.
__device__ __forceinline__ int find_tensor(const AdamArgs& a) {
    int k = 0;
    for (int j = 1; j < a.count; ++j)
        if (a.t[j].first <= blockIdx.x) k = j;
    return k;
}

template <typename P, typename G, bool Q8>
__global__ __launch_bounds__(kBlock) void k_adamw(AdamArgs a) {
    const AdamTensor& T = a.t[find_tensor(a)];
    P* p = static_cast<P*>(T.p);
    const G* g = static_cast<const G*>(T.g);
    const int64_t n = T.n, padded = adam_padded(n);
    const bool vec = T.vec != 0;
    const int64_t at = (int64_t)(blockIdx.x - T.first) * kAdamChunk + threadIdx.x * 4;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kAdamChunk; k += kBlock * 4) {
        const int64_t i = at + k;
        if (i >= padded) break;  // whole waves: 256 elements each
        float x[4], d[4], m[4], v[4], r[4];
        load4(p, i, n, vec, x);
        load4(g, i, n, vec, d);
        Moments<Q8>::load(T.state, n, i, m, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float ge = d[e] * a.grad_scale;
            const float mn = m[e] * a.beta1 + ge * a.one_beta1;
            const float vn = v[e] * a.beta2 + (ge * ge) * a.one_beta2;
            // |.| < inf is false for NaN too
            const bool ok = fabsf(mn) < INFINITY && vn < INFINITY;
            r[e] = sqrtf(ok ? vn : v[e]);
            const float step = (mn * a.rate) / (r[e] * a.fix + a.eps);
            if (ok) {
                x[e] = x[e] * a.keep - step;
                m[e] = mn;
                v[e] = vn;
            } else if (i + e < n) {
                bad = true;
            }
        }
        store4(p, i, n, vec, x);
        Moments<Q8>::store(T.state, n, i, m, v, r);
    }
    if (bad) atomicCAS(a.status, 0, -6);
}

template <bool Q8, bool WRITE>
__global__ __launch_bounds__(kBlock) void k_adamw_state(AdamArgs a) {
    const AdamTensor& T = a.t[find_tensor(a)];
    float* pm = static_cast<float*>(T.p);
    float* pv = static_cast<float*>(const_cast<void*>(T.g));
    const int64_t n = T.n, padded = adam_padded(n);
    const bool vec = T.vec != 0;
    const int64_t at = (int64_t)(blockIdx.x - T.first) * kAdamChunk + threadIdx.x * 4;
#pragma unroll
    for (int k = 0; k < kAdamChunk; k += kBlock * 4) {
        const int64_t i = at + k;
        if (i >= padded) break;
        float m[4], v[4], r[4];
        if constexpr (WRITE) {
            load4(pm, i, n, vec, m);
            load4(pv, i, n, vec, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = sqrtf(v[e]);
            Moments<Q8>::store(T.state, n, i, m, v, r);
        } else {
            Moments<Q8>::load(T.state, n, i, m, v);
            store4(pm, i, n, vec, m);
            store4(pv, i, n, vec, v);
        }
    }
}

}  // namespace

hipError_t launch_adamw(const AdamArgs& a, int64_t chunks, int32_t p_dtype, int32_t g_dtype,
                        int32_t state_kind, hipStream_t s) {
    const dim3 grid((uint32_t)chunks);
    const bool q8 = state_kind != 0;
#define HUGE_ADAM(P, G)                                             \
    do {                                                            \
        if (q8) k_adamw<P, G, true><<<grid, kBlock, 0, s>>>(a);     \
        else k_adamw<P, G, false><<<grid, kBlock, 0, s>>>(a);       \
    } while (0)
    if (p_dtype == kDtypeBf16) {
        if (g_dtype == kDtypeBf16) HUGE_ADAM(bf16_t, bf16_t);
        else HUGE_ADAM(bf16_t, float);
    } else {
        if (g_dtype == kDtypeBf16) HUGE_ADAM(float, bf16_t);
        else HUGE_ADAM(float, float);
    }
#undef HUGE_ADAM
    return hipGetLastError();
}

hipError_t launch_adamw_state(const AdamArgs& a, int64_t chunks, int32_t state_kind, bool write,
                              hipStream_t s) {
    const dim3 grid((uint32_t)chunks);
    if (state_kind != 0) {
        if (write) k_adamw_state<true, true><<<grid, kBlock, 0, s>>>(a);
        else k_adamw_state<true, false><<<grid, kBlock, 0, s>>>(a);
    } else {
        if (write) k_adamw_state<false, true><<<grid, kBlock, 0, s>>>(a);
        else k_adamw_state<false, false><<<grid, kBlock, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace huge
