// AdamW over many tensors, with moments as floats or in 8 bits.
//
// One pass: an element's parameter, gradient and moments are read, updated in
// registers and written.  A workgroup takes a chunk of kAdamChunk elements of one
// tensor, found in the launch's table (in the kernel's arguments); a wave takes
// 256 elements at a time, four a lane, which is one block of an 8-bit state: its
// scales are a maximum over the wave's registers.  Bound by memory: 129 million
// fp32 elements with fp32 moments take 680 us, 28 bytes each, 5.3 TB/s (a copy
// reaches 4.8).  256 million bf16 ones with moments in 8 bits move 10 bytes each and
// take 603 to 630 us, 4.2 TB/s: there the vector work of the exact roots and quotients and
// of the codes shows (0.4 of the time of four fp32 elements; the test of the new
// parameter is 3 to 5% of the whole).  Reading the
// moments out takes 466 us, 10 bytes an element, 5.5 TB/s.  A table of up to 64
// tensors goes in the kernel's arguments: four small tensors are one launch of 3 us.
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

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Four elements at i.  FULL: all there, at an address aligned for all four.
template <bool FULL, typename E>
__device__ __forceinline__ void load4(const E* __restrict__ p, int64_t i, int64_t n, float* v) {
    if constexpr (FULL) {
        const float4 q = load_chunk(p + i, 0);
        v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = 0.f;
            if (i + e < n) {
                if constexpr (sizeof(E) == 4) v[e] = p[i + e];
                else v[e] = __uint_as_float((uint32_t)p[i + e] << 16);
            }
        }
    }
}

template <bool FULL, typename E>
__device__ __forceinline__ void store4(E* __restrict__ p, int64_t i, int64_t n, const float* v) {
    if constexpr (FULL && sizeof(E) == 4) {
        store_chunk(p + i, 0, make_float4(v[0], v[1], v[2], v[3]));
    } else if constexpr (FULL) {
        *reinterpret_cast<bf16x4*>(p + i) =
            __builtin_convertvector((f32x4{v[0], v[1], v[2], v[3]}), bf16x4);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) {
                if constexpr (sizeof(E) == 4) p[i + e] = v[e];
                else p[i + e] = (bf16_t)float_to_bf16_bits(v[e]);
            }
    }
}

// Maximum over the wave of values >= 0, without LDS (as xor_add).
template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF,
                                                               0xF, false)));
}
__device__ __forceinline__ float wave_max(float v) {
    v = dpp_max<0xB1>(v);
    v = dpp_max<0x4E>(v);
    v = dpp_max<0x141>(v);
    v = dpp_max<0x140>(v);
    const int a = __float_as_int(v);
    const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    v = fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
    const int b = __float_as_int(v);
    const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return fmaxf(__int_as_float(q[0]), __int_as_float(q[1]));
}

// Roots and quotients to the nearest float by Markstein's method: the hardware's
// reciprocal (root), then a correction by the residual, which an fma gives without
// error.  A third of the instructions of sqrtf and of the division, which also
// serve subnormal numbers and infinities.
constexpr float kTiny = 0x1p-100f;  // above it, residuals are normal numbers

// sqrt(x) for x = 0 and x >= kTiny (what is between gives less than 2^-49).
__device__ __forceinline__ float root(float x) {
    const float y = __builtin_amdgcn_rsqf(fmaxf(x, kTiny));
    const float s = x * y;
    return __builtin_fmaf(__builtin_fmaf(-s, s, x), 0.5f * y, s);
}

// a / b for b >= 1e-30 and a quotient below 2^127.
__device__ __forceinline__ float quotient(float a, float b) {
    float y = __builtin_amdgcn_rcpf(b);
    y = __builtin_fmaf(__builtin_fmaf(-b, y, 1.0f), y, y);
    const float q = a * y;
    return __builtin_fmaf(__builtin_fmaf(-b, q, a), y, q);
}

// The moments of four elements at i (a multiple of 4) of a tensor of n.  `b`: the
// block of 256 that holds them.
template <bool Q8>
struct Moments;

template <>
struct Moments<false> {
    // the two arrays are padded to whole blocks: always four at a time
    static __device__ __forceinline__ void load(const uint8_t* state, int64_t padded, int64_t i,
                                                float* m, float* v) {
        const float* sm = reinterpret_cast<const float*>(state);
        load4<true>(sm, i, 0, m);
        load4<true>(sm + padded, i, 0, v);
    }
    static __device__ __forceinline__ void store(uint8_t* state, int64_t padded, int64_t i,
                                                 const float* m, const float* v, const float*) {
        float* sm = reinterpret_cast<float*>(state);
        store4<true>(sm, i, 0, m);
        store4<true>(sm + padded, i, 0, v);
    }
};

template <>
struct Moments<true> {
    static __device__ __forceinline__ float2* scales(uint8_t* state, int64_t padded, int64_t i) {
        return reinterpret_cast<float2*>(state + 2 * padded) + i / kAdamBlock;
    }
    static __device__ __forceinline__ void load(const uint8_t* state, int64_t padded, int64_t i,
                                                float* m, float* v) {
        const uint32_t q = *reinterpret_cast<const uint32_t*>(state + i);
        const uint32_t u = *reinterpret_cast<const uint32_t*>(state + padded + i);
        const float2 s = *scales(const_cast<uint8_t*>(state), padded, i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // codes of m are stored as q + 128
            const float k = ((float)((q >> (8 * e)) & 0xFFu) - 128.0f) * kInv127;
            m[e] = s.x * (k * fabsf(k));
            const float c = (float)((u >> (8 * e)) & 0xFFu) * kInv255;
            const float r = s.y * (c * c);
            v[e] = r * r;
        }
    }
    // r: sqrt(v), 0 past the end of the tensor (as m is).  Every lane of the wave
    // takes part: its 256 elements are one block.
    static __device__ __forceinline__ void store(uint8_t* state, int64_t padded, int64_t i,
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
            const float a = rintf(root(fabsf(m[e]) * is) * 127.0f);
            const float c = rintf(root(r[e] * it) * 255.0f);
            q = __builtin_amdgcn_cvt_pk_u8_f32(copysignf(a, m[e]) + 128.0f, e, q);
            u = __builtin_amdgcn_cvt_pk_u8_f32(fmaxf(c, r[e] > 0.f ? 1.0f : 0.0f), e, u);
        }
        *reinterpret_cast<uint32_t*>(state + i) = q;
        *reinterpret_cast<uint32_t*>(state + padded + i) = u;
        if ((threadIdx.x & 63) == 0) *scales(state, padded, i) = make_float2(s, t);
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

// One chunk, 1024 elements at a time.  FULL: all of it inside the tensor and aligned.
template <typename P, typename G, bool Q8, bool FULL>
__device__ __forceinline__ bool update_chunk(const AdamArgs& a, const AdamTensor& T, int64_t at) {
    P* p = static_cast<P*>(T.p);
    const G* g = static_cast<const G*>(T.g);
    const int64_t n = T.n, padded = adam_padded(n);
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kAdamChunk; k += kBlock * 4) {
        const int64_t i = at + k;
        if (!FULL && i >= padded) break;  // whole waves: 256 elements each
        float x[4], d[4], m[4], v[4], r[4];
        load4<FULL>(p, i, n, x);
        load4<FULL>(g, i, n, d);
        Moments<Q8>::load(T.state, padded, i, m, v);
        float mn[4], vn[4];
        uint32_t top = 0, low = 0xFFFFFFFFu;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float ge = d[e] * a.grad_scale;
            mn[e] = m[e] * a.beta1 + ge * a.one_beta1;
            vn[e] = v[e] * a.beta2 + (ge * ge) * a.one_beta2;
            // as integers, infinities and NaN are above all numbers; 0 - 1 is too
            const uint32_t mb = __float_as_uint(fabsf(mn[e])), vb = __float_as_uint(vn[e]);
            top = max(top, max(mb, vb));
            low = min(low, vb - 1u);
        }
        constexpr uint32_t kInf = 0x7F800000u, kLeast = (127u - 100u) << 23;
        // the new parameter: from half a step above the largest bf16 it would be infinite
        constexpr uint32_t kTop = sizeof(P) == 2 ? 0x7F7F8000u : kInf;
        float y[4];
        uint32_t far = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            r[e] = root(vn[e]);
            y[e] = x[e] * a.keep - quotient(mn[e] * a.rate, r[e] * a.fix + a.eps);
            far = max(far, __float_as_uint(fabsf(y[e])));
        }
        if (__ballot(top >= kInf || low < kLeast - 1u || far >= kTop) == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = mn[e], v[e] = vn[e], x[e] = y[e];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float rn = sqrtf(vn[e]);
                const float z = x[e] * a.keep - (mn[e] * a.rate) / (rn * a.fix + a.eps);
                // |.| < inf is false for NaN too
                const bool ok = fabsf(mn[e]) < INFINITY && vn[e] < INFINITY &&
                                fabsf(z) < __uint_as_float(kTop);
                r[e] = ok ? rn : sqrtf(v[e]);
                m[e] = ok ? mn[e] : m[e];
                v[e] = ok ? vn[e] : v[e];
                x[e] = ok ? z : x[e];
                bad |= !ok && (FULL || i + e < n);
            }
        }
        store4<FULL>(p, i, n, x);
        Moments<Q8>::store(T.state, padded, i, m, v, r);
    }
    return bad;
}

template <typename P, typename G, bool Q8>
__global__ __launch_bounds__(kBlock) void k_adamw(AdamArgs a) {
    const AdamTensor& T = a.t[find_tensor(a)];
    const int64_t first = (int64_t)(blockIdx.x - T.first) * kAdamChunk;
    const int64_t at = first + threadIdx.x * 4;
    const bool full = T.vec != 0 && first + kAdamChunk <= T.n;
    const bool bad = full ? update_chunk<P, G, Q8, true>(a, T, at)
                          : update_chunk<P, G, Q8, false>(a, T, at);
    if (bad) atomicCAS(a.status, 0, -6);
}

template <bool Q8, bool WRITE, bool FULL>
__device__ __forceinline__ void state_chunk(const AdamTensor& T, int64_t at) {
    float* pm = static_cast<float*>(T.p);
    float* pv = static_cast<float*>(const_cast<void*>(T.g));
    const int64_t n = T.n, padded = adam_padded(n);
#pragma unroll
    for (int k = 0; k < kAdamChunk; k += kBlock * 4) {
        const int64_t i = at + k;
        if (!FULL && i >= padded) break;
        float m[4], v[4], r[4];
        if constexpr (WRITE) {
            load4<FULL>(pm, i, n, m);
            load4<FULL>(pv, i, n, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = sqrtf(v[e]);
            Moments<Q8>::store(T.state, padded, i, m, v, r);
        } else {
            Moments<Q8>::load(T.state, padded, i, m, v);
            store4<FULL>(pm, i, n, m);
            store4<FULL>(pv, i, n, v);
        }
    }
}

template <bool Q8, bool WRITE>
__global__ __launch_bounds__(kBlock) void k_adamw_state(AdamArgs a) {
    const AdamTensor& T = a.t[find_tensor(a)];
    const int64_t first = (int64_t)(blockIdx.x - T.first) * kAdamChunk;
    if (T.vec != 0 && first + kAdamChunk <= T.n)
        state_chunk<Q8, WRITE, true>(T, first + threadIdx.x * 4);
    else
        state_chunk<Q8, WRITE, false>(T, first + threadIdx.x * 4);
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
