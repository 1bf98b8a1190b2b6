// Root-mean-square norm of rows with the residual's addition, in the rows' type or in
// 8 bits, its backward pass, and rows in 8 bits.
//
// A group of threads holds a row in registers, as in layer norm: the sum of the two
// inputs is rounded to the rows' type, stored and normalised as it was stored, so that
// the backward pass, which reads it again, sees the same row.  One reduction over the
// group, the sum of squares; every array is moved once.  Bound by memory (a copy reaches
// 4.75 TB/s): 60417 x 761 fp32 with a residual 131 us forward (5.6 TB/s), 155 us backward
// (4.7) and 5 us for the sums of the weight gradients; 65536 x 128 bf16, which stays in the
// caches, 13, 13 and 4 us.
//
// bf16 rows of whole aligned eights go 16 bytes a thread: 8 bits back to bf16, 1e6
// x 128, took 103 us with 8 bytes a thread where it takes 64 to 69.
//
// 8 bits: e4m3 codes under a power of two for each 32 columns, which eight threads
// hold: the largest of their absolute values, as integers, so that a NaN is above
// everything, gives the smallest power under which no code is above 448.  A code
// times a power of two is a bf16 number, so that what reads such rows widens them
// without another rounding.  1e6 x 128 bf16 into codes that are the formula's own (below):
// 87 to 95 us, 4.1 to 4.5 TB/s.  Rows as they are into codes: 1e6 x 128 bf16 68 to 71 us (5.5 TB/s),
// fp32 108 to 114 (5.8).
#include <type_traits>

#include "rows.hpp"

namespace huge {

namespace {

// The exponent of a block's scale from the bits of its largest absolute value; kNone
// where that is no number.
constexpr int kNone = 128;
__device__ __forceinline__ int scale_exponent(uint32_t big) {
    if (big >= 0x7F800000u) return kNone;
    // 448 = 1.75 2^8: one more above 1.75
    const int e = (int)((big + 0x1FFFFFu) >> 23) - 127 - 8;
    return e < kByteLeast ? kByteLeast : e;
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// W elements of a row: four, or eight of bf16 rows that are whole aligned eights (16 bytes).
template <int W>
struct Cells {
    float v[W];
};
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <int W, bool WHOLE, typename E>
__device__ __forceinline__ Cells<W> load_cells(const E* row, int c, int D) {
    Cells<W> r;
    if constexpr (W == 4) {
        const Few f = load_few<WHOLE>(row, c, D);
#pragma unroll
        for (int e = 0; e < 4; ++e) r.v[e] = f.v[e];
    } else if constexpr (sizeof(E) == 4) {
        const float4 p = load_chunk(row, 2 * c), q = load_chunk(row, 2 * c + 1);
        r = {{p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w}};
    } else {
        const u16x8 q = *reinterpret_cast<const u16x8*>(row + 8 * c);
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = __uint_as_float((uint32_t)q[e] << 16);
    }
    return r;
}

template <int W, bool WHOLE, typename E>
__device__ __forceinline__ void store_cells(E* row, int c, int D, const Cells<W>& r) {
    if constexpr (W == 4) {
        store_few<WHOLE>(row, c, D, Few{{r.v[0], r.v[1], r.v[2], r.v[3]}});
    } else if constexpr (sizeof(E) == 4) {
        store_chunk(row, 2 * c, make_float4(r.v[0], r.v[1], r.v[2], r.v[3]));
        store_chunk(row, 2 * c + 1, make_float4(r.v[4], r.v[5], r.v[6], r.v[7]));
    } else {
        const f32x8 q = {r.v[0], r.v[1], r.v[2], r.v[3], r.v[4], r.v[5], r.v[6], r.v[7]};
        *reinterpret_cast<bf16x8*>(row + 8 * c) = __builtin_convertvector(q, bf16x8);
    }
}

// The largest over the lanes that hold a block of 32 columns, W each: aligned, and all of
// them active (as xor_add).
template <int W>
__device__ __forceinline__ uint32_t max_of_block(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
    if constexpr (W == 4)
        v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));
    return v;
}

// W cells in 8 bits, and the exponent of their block's scale.  The lanes of a block call
// together; r is 0 past the row's end.
template <int W>
struct Bytes {
    uint32_t q[W / 4];
    int x;
};
template <int W>
__device__ __forceinline__ void codes_of(const Cells<W>& r, float mul, uint32_t* q) {
#pragma unroll
    for (int k = 0; k < W / 4; ++k) {
        const float* v = r.v + 4 * k;
        q[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[0] * mul, v[1] * mul, 0, false);
        q[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * mul, v[3] * mul, (int)q[k], true);
    }
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

template <int W>
__device__ __forceinline__ uint32_t largest_of_block(const Cells<W>& r) {
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < W; ++e) big = max(big, abs_bits(r.v[e]));
    return max_of_block<W>(big);
}
template <int W>
__device__ __forceinline__ Bytes<W> encode(const Cells<W>& r) {
    Bytes<W> o;
    o.x = scale_exponent(largest_of_block<W>(r));
    codes_of<W>(r, power(o.x == kNone ? 0 : -o.x), o.q);
    if (o.x == kNone) {
#pragma unroll
        for (int k = 0; k < W / 4; ++k) o.q[k] = 0x7F7F7F7Fu;  // NaN
    }
    return o;
}

// The same of numbers that are known within `near` of themselves, and whether another code or
// scale is that near.
template <int W>
__device__ __forceinline__ Bytes<W> encode_near(const Cells<W>& r, float near, bool& doubt) {
    const uint32_t big = largest_of_block<W>(r);
    Bytes<W> o;
    o.x = scale_exponent(big);
    // near 1.75 times a power of two, or the first that is no number
    const uint32_t steps = (uint32_t)(near * 0x1p24f) + 2u;  // floats within `near`
    doubt |= (big & 0x7FFFFFu) - 0x600000u + steps <= 2u * steps;
    doubt |= 0x7F800000u - big <= 2u * steps;
    uint32_t low[W / 4];
    const float mul = power(o.x == kNone ? 0 : -o.x);
    codes_of<W>(r, mul * (1.f + near), o.q);
    codes_of<W>(r, mul * (1.f - near), low);
#pragma unroll
    for (int k = 0; k < W / 4; ++k) {
        doubt |= o.x != kNone && o.q[k] != low[k];
        if (o.x == kNone) o.q[k] = 0x7F7F7F7Fu;  // NaN
    }
    return o;
}

// Stores them and, from the first cells of a block, its scale.
template <int W, bool WHOLE>
__device__ __forceinline__ void store_bytes(uint8_t* codes, uint8_t* scales, int c, int D,
                                            const Bytes<W>& o) {
    if (W * c >= D) return;
    if constexpr (W == 8) {
        *reinterpret_cast<u32x2*>(codes + 8 * c) = u32x2{o.q[0], o.q[1]};
    } else if constexpr (WHOLE) {
        *reinterpret_cast<uint32_t*>(codes + 4 * c) = o.q[0];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (4 * c + e < D) codes[4 * c + e] = (uint8_t)(o.q[0] >> (8 * e));
    }
    constexpr int kCells = kByteBlock / W;
    if (c % kCells == 0) scales[c / kCells] = (uint8_t)(o.x + 127);
}

// r + o, rounded to the rows' type.
template <typename E, int W>
__device__ __forceinline__ void add_rounded(Cells<W>& r, const Cells<W>& o) {
    typedef float Wide __attribute__((ext_vector_type(W)));
    Wide v;
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = r.v[e] + o.v[e];
    if constexpr (sizeof(E) == 2) {
        typedef __bf16 Near __attribute__((ext_vector_type(W)));
        v = __builtin_convertvector(__builtin_convertvector(v, Near), Wide);
    }
#pragma unroll
    for (int e = 0; e < W; ++e) r.v[e] = v[e];
}

// Row r0 + sub of rows at a stride: what all lanes share first, where 64-bit products are cheap;
// the lane's part is the same from turn to turn.
template <typename T>
__device__ __forceinline__ T* row_at(T* p, int64_t ld, int64_t r0, int sub) {
    return p + r0 * ld + sub * ld;
}

// The float next to v, towards zero where v is none, with its last bit set: rounded from
// there to the few bits of a code, a number is rounded as if it were rounded once.
__device__ __forceinline__ float to_odd(double v) {
    const float f = (float)v;
    const double back = (double)f;
    uint32_t b = __float_as_uint(f);
    if (back != v && b << 1 < 0xFF000000u) b = (b - (fabs(back) > fabs(v) ? 1u : 0u)) | 1u;
    return __uint_as_float(b);
}

// Sum over a row's threads in fp64, as row_sum; between two calls all of a workgroup's threads
// meet elsewhere.
template <int TPR>
__device__ __forceinline__ double row_sum64(double v, double* s) {
#pragma unroll
    for (int off = 1; off < (TPR < 64 ? TPR : 64); off <<= 1) v += __shfl_xor(v, off);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (s[0] + s[1]) + (s[2] + s[3]);
    }
    return v;
}

// 1 / sqrt(x), x > 0, from the hardware's within one unit by a Newton step, whose roundings
// are one and a half: half of that of x r0, and the last.  What the hardware takes for 0 is
// scaled before; an infinity's is 0 as it is.
__device__ __forceinline__ float inverse_root(float x) {
    const bool tiny = x < 0x1p-96f;
    const float v = tiny ? x * 0x1p64f : x;
    const float r0 = __builtin_amdgcn_rsqf(v);
    const float r = fmaf(0.5f * r0, fmaf(-(v * r0), r0, 1.f), r0);
    return x < INFINITY ? (tiny ? r * 0x1p32f : r) : r0;
}

// BYTES: a code that is next to where it changes would change with the last bits of fp32.
// Where one of a wave's is that near, its rows are formed in fp64 once more, so that all codes
// are those of the formula.  How near: n squares in sequence and over lanes are summed within
// n + 3 roundings with the mean and eps, rstd is within half of that and two, y within
// two more, and the test itself takes two.
template <int W, int TPR, int NV>
constexpr float near_of() {
    int levels = TPR > 64 ? 3 : 0;
    for (int k = 1; k < TPR && k < 64; k <<= 1) ++levels;
    return (0.5f * (NV * W + levels) + 8.f) * 0x1p-24f;
}

template <typename E, int W, int TPR, int NV, bool WHOLE, bool BYTES>
__global__ __launch_bounds__(kBlock) void k_rms(RmsArgs a) {
    __shared__ float s_sum[8];
    __shared__ double s_sum64[BYTES ? 4 : 1];
    int turn = 0;
    constexpr int kRows = kBlock / TPR;
    const int t = threadIdx.x % TPR, D = a.dim, chunks = (D + W - 1) / W;
    const E* x = static_cast<const E*>(a.x);
    const E* res = static_cast<const E*>(a.res);
    E* total = static_cast<E*>(a.total);
    const float inv = 1.0f / (float)D;
    const int sub = TPR == kBlock ? 0 : threadIdx.x / TPR;
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < a.n; r0 += (int64_t)gridDim.x * kRows) {
        const int64_t r = r0 + sub;
        if (r >= a.n) break;
        Cells<W> f[NV], o[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            f[i] = c < chunks ? load_cells<W, WHOLE>(row_at(x, a.ld_x, r0, sub), c, D) : Cells<W>{};
            if (res != nullptr) o[i] = c < chunks ? load_cells<W, WHOLE>(row_at(res, a.ld_res, r0, sub), c, D) : Cells<W>{};
        }
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            if (res != nullptr) {
                add_rounded<E>(f[i], o[i]);
                if (c < chunks) store_cells<W, WHOLE>(row_at(total, a.ld_total, r0, sub), c, D, f[i]);
            }
#pragma unroll
            for (int e = 0; e < W; ++e) sq = fmaf(f[i].v[e], f[i].v[e], sq);
        }
        const float rstd = inverse_root(row_sum<TPR>(sq, s_sum, turn) * inv + a.eps);
        if (t == 0 && a.rstd != nullptr) a.rstd[r] = rstd;
        if constexpr (!BYTES) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = t + TPR * i;
                if (c >= chunks) continue;
                const Cells<W> g = load_cells<W, WHOLE>(a.gamma, c, D);
#pragma unroll
                for (int e = 0; e < W; ++e) f[i].v[e] = f[i].v[e] * rstd * g.v[e];
                store_cells<W, WHOLE>(row_at(static_cast<E*>(a.y), a.ld_y, r0, sub), c, D, f[i]);
            }
        } else {
            uint8_t* codes = row_at(a.codes, a.ld_codes, r0, sub);
            uint8_t* scales = row_at(a.scales, a.ld_scales, r0, sub);
            Bytes<W> q[NV];
            constexpr float kNear = near_of<W, TPR, NV>();
            bool doubt = false;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = t + TPR * i;
                const Cells<W> g = c < chunks ? load_cells<W, WHOLE>(a.gamma, c, D) : Cells<W>{};
                Cells<W> y;
#pragma unroll
                for (int e = 0; e < W; ++e) y.v[e] = f[i].v[e] * rstd * g.v[e];
                q[i] = encode_near<W>(y, kNear, doubt);
            }
            bool again;
            if constexpr (TPR > 64) again = __syncthreads_or(doubt);
            else again = __ballot(doubt) != 0;
            if (again) {
                double sq64 = 0.0;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        sq64 = fma((double)f[i].v[e], (double)f[i].v[e], sq64);
                        asm volatile("" : "+v"(f[i].v[e]));
                    }
                // 1 / D and the root by Newton's method from what the hardware has.  Few registers:
                // what is widened is not kept, and gamma is read here again
                double inv64 = (double)inv;
                inv64 = fma(inv64, fma(-(double)D, inv64, 1.0), inv64);
                const double x64 = fma(row_sum64<TPR>(sq64, s_sum64), inv64, (double)a.eps);
                double rstd64 = __builtin_amdgcn_rsq(x64);
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    rstd64 = fma(0.5 * rstd64, fma(-x64 * rstd64, rstd64, 1.0), rstd64);
                if (rstd == 0.f) rstd64 = 0.0;  // the sum passed fp32, whatever row calls for fp64
                uint64_t gamma_at = reinterpret_cast<uint64_t>(a.gamma);
                asm volatile("" : "+s"(gamma_at));
                const float* gamma = (const float*)(const __attribute__((address_space(1))) float*)gamma_at;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = t + TPR * i;
                    const Cells<W> g = c < chunks ? load_cells<W, WHOLE>(gamma, c, D) : Cells<W>{};
                    Cells<W> y;
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        float ge = g.v[e];
                        asm volatile("" : "+v"(ge));  // one after the other
                        y.v[e] = to_odd((double)f[i].v[e] * rstd64 * (double)ge);
                    }
                    q[i] = encode<W>(y);
                }
            }
#pragma unroll
            for (int i = 0; i < NV; ++i)
                store_bytes<W, WHOLE>(codes, scales, t + TPR * i, D, q[i]);
        }
    }
}

template <typename E, int W, int TPR, int NV, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_rms_backward(RmsArgs a) {
    __shared__ float s_sum[8];
    int turn = 0;
    constexpr int kRows = kBlock / TPR;
    constexpr int kHeld = TPR < 64 ? TPR : 64;  // lanes of a wave that hold different columns
    const int t = threadIdx.x % TPR, D = a.dim, chunks = (D + W - 1) / W;
    const E* x = static_cast<const E*>(a.x);
    const E* dy = static_cast<const E*>(a.dy);
    const E* res = static_cast<const E*>(a.res);
    E* dx = static_cast<E*>(a.y);
    const float inv = 1.0f / (float)D;
    Cells<W> g[NV], dg[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = t + TPR * i;
        g[i] = c < chunks ? load_cells<W, WHOLE>(a.gamma, c, D) : Cells<W>{};
        dg[i] = Cells<W>{};
    }
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; r < a.n;
         r += (int64_t)gridDim.x * kRows) {
        const float rstd = a.rstd[r];
        Cells<W> z[NV], d[NV], o[NV];
        float along = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            const bool in = c < chunks;
            z[i] = in ? load_cells<W, WHOLE>(x + r * a.ld_x, c, D) : Cells<W>{};
            d[i] = in ? load_cells<W, WHOLE>(dy + r * a.ld_dy, c, D) : Cells<W>{};
            o[i] = in && res != nullptr ? load_cells<W, WHOLE>(res + r * a.ld_res, c, D) : Cells<W>{};
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int e = 0; e < W; ++e) {
                z[i].v[e] *= rstd;
                dg[i].v[e] = fmaf(d[i].v[e], z[i].v[e], dg[i].v[e]);
                d[i].v[e] *= g[i].v[e];
                along = fmaf(d[i].v[e], z[i].v[e], along);
            }
        }
        if (dx == nullptr) continue;
        along = row_sum<TPR>(along, s_sum, turn) * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            if (c >= chunks) continue;
#pragma unroll
            for (int e = 0; e < W; ++e)
                d[i].v[e] = fmaf(rstd, d[i].v[e] - z[i].v[e] * along, o[i].v[e]);
            store_cells<W, WHOLE>(dx + r * a.ld_y, c, D, d[i]);
        }
    }
    if (a.partial == nullptr) return;
    // the groups of a wave, then the waves
    __shared__ float s_part[TPR <= 64 ? 4 * kHeld * NV * W : 1];
    float* out = a.partial + (int64_t)blockIdx.x * D;
    if constexpr (TPR <= 64) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < W; ++e) {
                float v = dg[i].v[e];
#pragma unroll
                for (int off = TPR; off < 64; off <<= 1) v += __shfl_xor(v, off);
                if (lane < kHeld) s_part[((wave * NV + i) * W + e) * kHeld + lane] = v;
            }
        __syncthreads();
        for (int j = threadIdx.x; j < D; j += kBlock) {
            const int c = j / W, at = ((c / TPR) * W + j % W) * kHeld + c % TPR;
            constexpr int kWave = NV * W * kHeld;
            out[j] = (s_part[at] + s_part[kWave + at]) +
                     (s_part[2 * kWave + at] + s_part[3 * kWave + at]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = t + TPR * i;
            if (c >= chunks) continue;
#pragma unroll
            for (int e = 0; e < W; ++e)
                if (W * c + e < D) out[c * W + e] = dg[i].v[e];
        }
    }
}

// Column sums of `partial`: a workgroup takes 8 columns, 32 threads each.
__global__ __launch_bounds__(kBlock) void k_rms_reduce(const float* __restrict__ partial,
                                                       int blocks, int dim,
                                                       float* __restrict__ dgamma) {
    __shared__ float s[32][9];
    const int col = blockIdx.x * 8 + (threadIdx.x & 7), lane = threadIdx.x >> 3;
    float v = 0.f;
    if (col < dim) {
#pragma unroll 8
        for (int b = lane; b < blocks; b += 32) v += partial[(int64_t)b * dim + col];
    }
    s[lane][threadIdx.x & 7] = v;
    __syncthreads();
    if (lane == 0 && col < dim) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) sum += s[k][threadIdx.x & 7];
        dgamma[col] = sum;
    }
}

// Rows into 8 bits: a thread takes W columns, in the order of rows' blocks of 32.
template <typename E, int W, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_to_bytes(RmsArgs a) {
    constexpr int kCells = kByteBlock / W;
    const int D = a.dim, blocks = (D + kByteBlock - 1) / kByteBlock;
    const int64_t all = a.n * blocks;
    for (int64_t b = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kCells; b < all;
         b += (int64_t)gridDim.x * kBlock / kCells) {
        const int64_t r = b / blocks;
        const int c = (int)(b % blocks) * kCells + threadIdx.x % kCells;
        const Cells<W> f =
            W * c < D ? load_cells<W, WHOLE>(static_cast<const E*>(a.x) + r * a.ld_x, c, D) : Cells<W>{};
        store_bytes<W, WHOLE>(a.codes + r * a.ld_codes, a.scales + r * a.ld_scales, c, D,
                              encode<W>(f));
    }
}

// ... and back: a thread takes W columns.
template <typename E, int W, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_from_bytes(RmsArgs a) {
    constexpr int kCells = kByteBlock / W;
    const int D = a.dim, chunks = (D + W - 1) / W;
    const int64_t all = a.n * chunks;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < all;
         i += (int64_t)gridDim.x * kBlock) {
        const int64_t r = i / chunks;
        const int c = (int)(i % chunks);
        const uint8_t* row = a.codes + r * a.ld_codes;
        uint32_t q[W / 4] = {};
        if constexpr (W == 8) {
            const u32x2 v = reinterpret_cast<const u32x2*>(row)[c];
            q[0] = v.x, q[1] = v.y;
        } else if constexpr (WHOLE) {
            q[0] = reinterpret_cast<const uint32_t*>(row)[c];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (4 * c + e < D) q[0] |= (uint32_t)row[4 * c + e] << (8 * e);
        }
        const float mul = byte_scale(a.scales[r * a.ld_scales + c / kCells]);
        Cells<W> f;
#pragma unroll
        for (int k = 0; k < W / 4; ++k) {
            f.v[4 * k] = __builtin_amdgcn_cvt_f32_fp8((int)q[k], 0) * mul;
            f.v[4 * k + 1] = __builtin_amdgcn_cvt_f32_fp8((int)q[k], 1) * mul;
            f.v[4 * k + 2] = __builtin_amdgcn_cvt_f32_fp8((int)q[k], 2) * mul;
            f.v[4 * k + 3] = __builtin_amdgcn_cvt_f32_fp8((int)q[k], 3) * mul;
        }
        store_cells<W, WHOLE>(static_cast<E*>(a.y) + r * a.ld_y, c, D, f);
    }
}

template <typename E, int W, int TPR, int NV, bool WHOLE>
void rms_one(const RmsArgs& a, bool backward, hipStream_t s) {
    const int64_t rows = kBlock / TPR, need = (a.n + rows - 1) / rows;
    // into 8 bits vector instructions show, and what comes before the loop is done for several
    // rows (1e6 x 128 bf16 and back: 158 us, 168 with up to 65536 workgroups); else memory
    // bounds, and one row a group is a little faster (200000 x 256 fp32 both ways 303 and 310)
    const int64_t most = a.codes != nullptr ? 8192 : 65536;
    const dim3 grid((uint32_t)(need < most ? need : most));
    if (backward)
        k_rms_backward<E, W, TPR, NV, WHOLE>
            <<<dim3((uint32_t)norm_blocks(a.n, a.dim)), kBlock, 0, s>>>(a);
    else if (a.codes != nullptr)
        k_rms<E, W, TPR, NV, WHOLE, true><<<grid, kBlock, 0, s>>>(a);
    else
        k_rms<E, W, TPR, NV, WHOLE, false><<<grid, kBlock, 0, s>>>(a);
}

template <typename E, int W, bool WHOLE>
hipError_t rms_shape(const RmsArgs& a, bool backward, hipStream_t s) {
    const NormShape p = norm_shape((a.dim + W - 1) / W);
#define HUGE_RMS_CASE(T, N)                           \
    case (T) * 64 + (N):                              \
        rms_one<E, W, T, N, WHOLE>(a, backward, s);   \
        return hipGetLastError();
    switch (p.tpr * 64 + p.nv) {
        HUGE_RMS_CASE(8, 1)
        HUGE_RMS_CASE(16, 1)
        HUGE_RMS_CASE(32, 1)
        HUGE_RMS_CASE(64, 1)
        HUGE_RMS_CASE(64, 2)
        HUGE_RMS_CASE(64, 4)
        HUGE_RMS_CASE(256, 2)
        HUGE_RMS_CASE(256, 4)
    }
    if constexpr (W == 4) {
        switch (p.tpr * 64 + p.nv) { HUGE_RMS_CASE(256, 8) }
    }
#undef HUGE_RMS_CASE
    return hipErrorInvalidValue;
}

template <typename E>
hipError_t rms_dispatch(const RmsArgs& a, bool backward, hipStream_t s) {
    if constexpr (sizeof(E) == 2)
        if (a.eights) return rms_shape<E, 8, true>(a, backward, s);
    return a.vec ? rms_shape<E, 4, true>(a, backward, s) : rms_shape<E, 4, false>(a, backward, s);
}

template <typename E>
hipError_t bytes_dispatch(const RmsArgs& a, bool back, hipStream_t s) {
    const int w = a.eights ? 8 : 4;
    const int64_t work = back ? a.n * ((a.dim + w - 1) / w)
                              : a.n * ((a.dim + kByteBlock - 1) / kByteBlock) * (kByteBlock / w);
    const int64_t need = (work + kBlock - 1) / kBlock;
    const dim3 grid((uint32_t)(need < 65536 ? need : 65536));
    if (back) {
        if (a.eights) k_from_bytes<E, 8, true><<<grid, kBlock, 0, s>>>(a);
        else if (a.vec) k_from_bytes<E, 4, true><<<grid, kBlock, 0, s>>>(a);
        else k_from_bytes<E, 4, false><<<grid, kBlock, 0, s>>>(a);
    } else {
        if (a.eights) k_to_bytes<E, 8, true><<<grid, kBlock, 0, s>>>(a);
        else if (a.vec) k_to_bytes<E, 4, true><<<grid, kBlock, 0, s>>>(a);
        else k_to_bytes<E, 4, false><<<grid, kBlock, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rms(const RmsArgs& a, hipStream_t s) {
    return a.dtype == kDtypeBf16 ? rms_dispatch<bf16_t>(a, false, s)
                                 : rms_dispatch<float>(a, false, s);
}

hipError_t launch_rms_backward(const RmsArgs& a, float* dgamma, hipStream_t s) {
    if (a.n > 0) {
        const hipError_t e = a.dtype == kDtypeBf16 ? rms_dispatch<bf16_t>(a, true, s)
                                                   : rms_dispatch<float>(a, true, s);
        if (e != hipSuccess) return e;
    }
    if (dgamma == nullptr) return hipSuccess;
    k_rms_reduce<<<dim3((uint32_t)((a.dim + 7) / 8)), kBlock, 0, s>>>(
        a.partial, norm_blocks(a.n, a.dim), a.dim, dgamma);
    return hipGetLastError();
}

hipError_t launch_to_bytes(const RmsArgs& a, hipStream_t s) {
    return a.dtype == kDtypeBf16 ? bytes_dispatch<bf16_t>(a, false, s)
                                 : bytes_dispatch<float>(a, false, s);
}

hipError_t launch_from_bytes(const RmsArgs& a, hipStream_t s) {
    return a.dtype == kDtypeBf16 ? bytes_dispatch<bf16_t>(a, true, s)
                                 : bytes_dispatch<float>(a, true, s);
}

}  // namespace huge
