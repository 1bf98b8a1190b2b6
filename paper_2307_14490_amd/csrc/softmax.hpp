// The exact softmax loss over a large vocabulary and its gradient, without the
// logits in memory.
//
// With S = H W' + bias, the loss needs lse_i = log sum_j exp S_ij, and the gradient
// G = c (exp(S - lse) - onehot) only in the products G W and G' H.  Each of the
// three passes forms a 32 x 32 tile of S on the matrix cores, uses it in
// registers and drops it: the loss keeps a running maximum and sum per row, the
// two gradients multiply the tile at once.  S is formed three times in all, which
// at the widths of embeddings costs less than a round trip of its elements
// through memory: 2 D flops are 0.06 clocks of a CU at D = 128, the 2 + 2 bytes of
// an element kept in half width 0.4 at the rate of a copy.
//
// Both gradients are one kernel: X are the rows whose gradient is formed (XB tiles
// of 32 per wave, held in registers), Y the rows that are summed over.  A tile is
// computed with Y as the rows and X as the columns of the product, so that a lane
// holds 16 elements of one X row: sums, maxima and scales per X row need no
// exchange between lanes, and the tile as it lies is the second operand of the
// product with Y' (whose operand holds Y's rows in the order in which the first
// product leaves them).
//
// Operands are packed before, in records of 32 rows: a header with the rows'
// terms, the R form (rows as they enter S) and the T form (rows as they enter the
// second product), each 1 KB block one operand of a 32x32x16 product in lane order.
// A workgroup streams Y's records through two LDS buffers (copied by the loads
// that write LDS, while the other buffer is used); reads of an operand are 1 KB in
// a row and meet no bank conflict.
//
// Precision.  bf16 rows enter as they are, and the tile is rounded to bf16 after
// the label is subtracted, so that a probability near one keeps its small
// complement: an error of 2^-8 of each term at most, as in the rounding of the
// result (2.0e-3 to 2.3e-3 of the gradients' norm in all, of which that rounding
// alone is 1.7e-3).  Two bf16 parts of the tile would leave the latter only, for a
// second product twice as long: 4096 x 1e6 x 128 3731 -> 5197 us, 100003 x 1000 x
// 128 164 -> 199, 4096 x 50021 x 384 728 -> 904.  fp32 rows are scaled by a power of two per row and split into two fp16
// parts, hi + lo (22 bits of an element within 2^-17 of the row's largest, and
// 2^-40 of that for smaller ones), and the products hi hi + hi lo + lo hi are
// summed in fp32; the tile is split the same way under a scale per X row that
// follows the largest element so far.  Maxima, sums and gradients are fp32.
//
// Two pairs of calls are made of these kernels: the loss and its gradient
// (k_softmax.hip), and log probabilities, which also need the entropy and each tile's
// largest logit, with the gradient of weights of either sign (k_answer.hip).  ANSWER
// marks what the second pair adds.  Its bf16 gradients hold G in fp16 under a scale per X
// row, as those of fp32 rows do: weights of either sign cancel in the sums, where the
// rounding to bf16 would show (2.3e-3 to 2.5e-3 of the norm, 1.7e-3 with fp16, which is the
// result's own rounding; 100003 x 1000 x 128 149 us and 168).  There a class that is out has the finite term
// kFloor (in gradients kGradFloor), so that the product of a vanishing probability and its
// logarithm is 0, and the running maximum starts at kLeast, far above that: a row without
// classes sums to 0.
#pragma once

#include <math.h>

#include <type_traits>

#include "device.hpp"
#include "head.hpp"

namespace huge {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kFloor = -1e30f, kLeast = -1e28f;
// The term in gradients, where an element is a vanishing probability times its logarithm
// times a weight: 0 for weights up to 1e18, as that product stays finite.  Far below what logits
// may be (1e9) all the same.
constexpr float kGradFloor = -1e20f;

// Element types: how rows are split, and the product of two operands.
template <typename E>
struct Kind;

template <>
struct Kind<bf16_t> {
    using Vec = bf16x8;
    static constexpr int kParts = 1;
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ f32x16 mfma(Vec a, Vec b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};

template <>
struct Kind<float> {
    using Vec = f16x8;
    static constexpr int kParts = 2;
    static constexpr bool kScaled = true;
    static __device__ __forceinline__ f32x16 mfma(Vec a, Vec b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};

template <typename E>
struct Operand {
    typename Kind<E>::Vec p[Kind<E>::kParts];
};

// The parts of eight values: each the nearest to what the ones before leave.
template <typename E>
__device__ __forceinline__ Operand<E> split(f32x8 v) {
    Operand<E> r;
    r.p[0] = __builtin_convertvector(v, typename Kind<E>::Vec);
    if constexpr (Kind<E>::kParts == 2)
        r.p[1] = __builtin_convertvector(v - __builtin_convertvector(r.p[0], f32x8),
                                         typename Kind<E>::Vec);
    return r;
}

// c + a b.
template <typename E>
__device__ __forceinline__ f32x16 product(const Operand<E>& a, const Operand<E>& b, f32x16 c) {
    if constexpr (Kind<E>::kParts == 2) {
        c = Kind<E>::mfma(a.p[1], b.p[0], c);
        c = Kind<E>::mfma(a.p[0], b.p[1], c);
    }
    return Kind<E>::mfma(a.p[0], b.p[0], c);
}

// The second product of answers' bf16 gradients: halves, whose bits take the place of an
// operand's.
template <typename E, bool HALF_BITS>
__device__ __forceinline__ f32x16 second_product(const Operand<E>& a, const Operand<E>& b, f32x16 c) {
    if constexpr (HALF_BITS)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a.p[0]),
                                                      __builtin_bit_cast(f16x8, b.p[0]), c, 0, 0, 0);
    else
        return product<E>(a, b, c);
}
template <typename E, bool HALF_BITS>
__device__ __forceinline__ Operand<E> second_split(f32x8 v) {
    if constexpr (HALF_BITS) {
        Operand<E> r;
        r.p[0] = __builtin_bit_cast(typename Kind<E>::Vec, __builtin_convertvector(v, f16x8));
        return r;
    } else {
        return split<E>(v);
    }
}

// Row of a product's register i in lane half h (the column is lane % 32).
__device__ __forceinline__ int tile_row(int i, int h) { return 8 * (i / 4) + 4 * h + i % 4; }

// A record's header: 32 of each.
constexpr int kHeader = 1024;
enum Field : int {
    kTerm = 0,    // classes: bias, -inf where the class is out
    kTerm2 = 1,   // the same times log2(e); rows: (log weight - lse) log2(e), -inf without a loss
    kMul = 2,     // fp32, and the T form of answers: what the packed row is to be multiplied by
    kLabel = 3,   // rows: label (int32), -1 without a loss
    kWeight = 4,  // rows: weight
    kSlope = 5,   // rows of weights of either sign: an element is p (kSlope log2 p + kCoef),
    kCoef = 6,    // less kWeight at the label
};
__device__ __forceinline__ const float* field(const uint8_t* rec, Field f) {
    return reinterpret_cast<const float*>(rec) + 32 * f;
}

// Bytes of a record: `forms` forms of nfrag operands and kParts parts.
__host__ __device__ constexpr int record_bytes(int nfrag, int parts, int forms) {
    return kHeader + forms * parts * nfrag * 1024;
}

// Operand f of the form that starts at `form`, whose parts are nfrag operands apart.
template <typename E>
__device__ __forceinline__ Operand<E> load_operand(const uint8_t* form, int f, int nfrag,
                                                   int lane) {
    using Vec = typename Kind<E>::Vec;
    Operand<E> r;
#pragma unroll
    for (int k = 0; k < Kind<E>::kParts; ++k)
        r.p[k] = reinterpret_cast<const Vec*>(form)[(k * nfrag + f) * 64 + lane];
    return r;
}

// The 16 values that go with a lane's elements of a tile, from a header field.  LDS
// is read here, as everywhere in the loops below, as vector types: a read of
// another type is taken to alias the copy in flight, and waits for it.
__device__ __forceinline__ f32x4 row_four(const uint8_t* rec, Field f, int half, int g) {
    return reinterpret_cast<const f32x4*>(field(rec, f))[2 * g + half];
}
__device__ __forceinline__ f32x16 row_values(const uint8_t* rec, Field f, int half) {
    f32x16 r;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 q = row_four(rec, f, half, g);
        r[4 * g] = q.x, r[4 * g + 1] = q.y, r[4 * g + 2] = q.z, r[4 * g + 3] = q.w;
    }
    return r;
}

// Sum of a lane's elements of a tile, in pairs: added one by one to a running sum,
// each would be rounded at the size of that.
__device__ __forceinline__ float sum16(f32x16 v) {
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = v[i] + v[i + 8];
    return ((s[0] + s[4]) + (s[2] + s[6])) + ((s[1] + s[5]) + (s[3] + s[7]));
}

// A lane's value of a header field (its row is the lane's column).
__device__ __forceinline__ int32_t lane_label(const uint8_t* rec, int lane) {
    typedef int32_t one __attribute__((ext_vector_type(2)));
    const one v = reinterpret_cast<const one*>(field(rec, kLabel))[(lane & 31) >> 1];
    return lane & 1 ? v.y : v.x;
}

__device__ __forceinline__ void set_status(int32_t* status, int32_t code) {
    atomicCAS(status, 0, code);
}

// ---------------------------------------------------------------------------
// Packing
// ---------------------------------------------------------------------------
// The largest magnitude of p (slope log2 p + coef), less weight, over p in 0 .. 1: p log2 p
// is within 1 / (e ln 2) = 0.5307.
__device__ __forceinline__ float element_bound(float slope, float coef, float weight) {
    return 0.54f * fabsf(slope) + fabsf(coef) + fabsf(weight);
}

struct PackArgs {
    const void* m;
    int64_t ld, first, count;  // rows first .. first + count of the matrix
    int64_t tiles;
    uint8_t* out;
    bool classes;              // or rows
    bool vec;                  // four elements at a time
    const uint8_t* scales;     // classes in 8 bits: m holds their codes
    int64_t ld_scales;
};

constexpr int kPackCols = 256;

// Four elements of a row at a column, 0 past its end.
template <typename E>
__device__ __forceinline__ float4 load_cols(const E* row, int col, int dim, bool vec) {
    if (col >= dim) return zero4();
    if (vec) return load_chunk(row + col, 0);
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(E) == 4) v[e] = row[col + e];
        else v[e] = __uint_as_float((uint32_t)row[col + e] << 16);
    }
    return make_float4(v[0], v[1], v[2], v[3]);
}

// The same of a row in 8 bits, the columns being whole fours.
__device__ __forceinline__ float4 load_code_cols(const uint8_t* row, const uint8_t* scales, int col,
                                                 int dim, bool vec) {
    if (col >= dim) return zero4();
    uint32_t q;
    if (vec) q = *reinterpret_cast<const uint32_t*>(row + col);
    else q = row[col] | row[col + 1] << 8 | row[col + 2] << 16 | (uint32_t)row[col + 3] << 24;
    const float mul = byte_scale(scales[col / kByteBlock]);
    return make_float4(__builtin_amdgcn_cvt_f32_fp8((int)q, 0) * mul,
                       __builtin_amdgcn_cvt_f32_fp8((int)q, 1) * mul,
                       __builtin_amdgcn_cvt_f32_fp8((int)q, 2) * mul,
                       __builtin_amdgcn_cvt_f32_fp8((int)q, 3) * mul);
}

__device__ __forceinline__ float max4(float m, float4 v) {
    return fmaxf(fmaxf(fmaxf(m, fabsf(v.x)), fmaxf(fabsf(v.y), fabsf(v.z))), fabsf(v.w));
}

// A workgroup packs a record, 256 columns at a time through LDS; eight threads
// read a row.  Bound by memory: 1e6 x 128 bf16 into both forms 142 us, 768 bytes a
// row, 5.4 TB/s.
template <typename E, bool ANSWER, bool CODES>
__global__ __launch_bounds__(kBlock) void k_sm_pack(SoftmaxArgs a, PackArgs w, PackArgs h,
                                                    int nfrag, int forms, int64_t first) {
    constexpr int kParts = Kind<E>::kParts;
    using Vec = typename Kind<E>::Vec;
    __shared__ float s[32][kPackCols + 4];
    __shared__ bool s_out[32];
    __shared__ float s_mul[32];
    const int64_t block = first + blockIdx.x;
    const bool second = block >= w.tiles;
    const PackArgs& k = second ? h : w;
    const int64_t tile = second ? block - w.tiles : block;
    uint8_t* rec = k.out + tile * record_bytes(nfrag, kParts, forms);
    float* head = reinterpret_cast<float*>(rec);
    if (threadIdx.x < 32) {
        const int r = threadIdx.x;
        const int64_t i = tile * 32 + r;
        bool out = i >= k.count;
        float term = -INFINITY, term2 = -INFINITY, weight = 0.f;
        int32_t label = -1;
        if (k.classes) {
            if (!out) term = a.bias == nullptr ? 0.f : a.bias[k.first + i];
            if constexpr (ANSWER) {
                out = term < kLeast;
                if (out) term = forms == 2 ? kGradFloor : kFloor;
            } else {
                out = term == -INFINITY;
            }
            term2 = term * kLog2e;
        } else if (ANSWER && forms == 2) {
            float coef = 0.f, slope = 0.f;
            term2 = kFloor;
            if (!out) {
                label = a.labels == nullptr ? -1 : a.labels[i];
                if (label < -1 || label >= a.classes) {
                    set_status(a.status, -2);
                    label = -1;
                }
                if (label >= 0 && a.bias != nullptr && a.bias[label] < kLeast) label = -1;
                const float dl = a.dlogp == nullptr || label < 0 ? 0.f : a.dlogp[i];
                const float de = a.dentropy == nullptr ? 0.f : a.dentropy[i];
                const float lse = a.lse[i];
                out = (dl == 0.f && de == 0.f) || lse == -INFINITY;
                if (out) {
                    label = -1;
                } else {
                    // rounded once: it reaches the logarithm of every element of the row
                    term2 = (float)((double)lse * -1.4426950408889634);
                    weight = -dl;
                    coef = de == 0.f ? -dl : -fmaf(de, a.entropy[i], dl);
                    slope = de * -0.69314718055994531f;
                }
            }
            head[32 * kSlope + r] = slope;
            head[32 * kCoef + r] = coef;
        } else if (!out && forms == 2) {
            label = a.labels[i];
            weight = a.weight == nullptr ? 1.f : a.weight[i];
            const bool bad_y = label < -1 || label >= a.classes;
            const bool bad_c = !(weight >= 0.f && weight < INFINITY);
            if (bad_y) set_status(a.status, -2);
            else if (bad_c) set_status(a.status, -3);
            if (bad_y || bad_c || label < 0 || weight == 0.f ||
                (a.bias != nullptr && a.bias[label] == -INFINITY)) {
                label = -1;
                weight = 0.f;
                out = true;
            } else {
                // rounded once: it reaches the exponent of every element of the row
                term2 = (float)(((double)logf(weight) - (double)a.lse[i]) * 1.4426950408889634);
            }
        }
        s_out[r] = out;
        head[32 * kTerm + r] = term;
        head[32 * kTerm2 + r] = term2;
        reinterpret_cast<int32_t*>(head)[32 * kLabel + r] = label;
        head[32 * kWeight + r] = weight;
    }
    __syncthreads();
    const int row = threadIdx.x >> 3, j0 = (threadIdx.x & 7) * 4;
    const E* m = static_cast<const E*>(k.m) + (k.first + tile * 32 + row) * k.ld;
    const bool out = s_out[row];
    const int64_t at = k.first + tile * 32 + row;
    auto cols = [&](int col) {
        if constexpr (CODES)
            if (!second)
                return load_code_cols(static_cast<const uint8_t*>(k.m) + at * k.ld,
                                      k.scales + at * k.ld_scales, col, a.dim, k.vec);
        return load_cols(m, col, a.dim, k.vec);
    };
    // answers' T form is halves of rows under a scale that a record shares: G's elements then
    // need one factor for a tile, where a scale per row would be one for each
    constexpr bool kHalfT = ANSWER && !Kind<E>::kScaled;
    float half_mul = 1.f;
    if (Kind<E>::kScaled || (kHalfT && forms == 2)) {
        float big = 0.f;
        if (!out)
            for (int col = j0; col < a.dim; col += 32) big = max4(big, cols(col));
        big = fmaxf(big, __shfl_xor(big, 1));
        big = fmaxf(big, __shfl_xor(big, 2));
        big = fmaxf(big, __shfl_xor(big, 4));
        auto exponent = [](float v) {
            // v < 2^e: scaled by 2^(15 - e) the row is below 2^15
            const int e = v > 0.f && v < INFINITY ? __builtin_amdgcn_frexp_expf(v) : 0;
            return e < -100 ? -100 : e;
        };
        if constexpr (Kind<E>::kScaled) {
            if ((threadIdx.x & 7) == 0) {
                const int e = exponent(big);
                s_mul[row] = ldexpf(1.f, 15 - e);
                head[32 * kMul + row] = ldexpf(1.f, e - 15);
            }
            __syncthreads();
        } else {
            if ((threadIdx.x & 7) == 0) s_mul[row] = big;
            __syncthreads();
            // an infinity counts for nothing: its row's products are no numbers in any scale
            float most = 0.f;
#pragma unroll 8
            for (int r = 0; r < 32; ++r) most = s_mul[r] < INFINITY ? fmaxf(most, s_mul[r]) : most;
            const int e = exponent(most);
            half_mul = ldexpf(1.f, 15 - e);
            if (threadIdx.x < 32) head[32 * kMul + threadIdx.x] = ldexpf(1.f, e - 15);
        }
    }
    const float mul = Kind<E>::kScaled ? s_mul[row] : 1.f;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int nd = nfrag / 2;
    Vec* form = reinterpret_cast<Vec*>(rec + kHeader);
    for (int c0 = 0; c0 < 16 * nfrag; c0 += kPackCols) {
        for (int col = j0; col < kPackCols; col += 32)
            *reinterpret_cast<float4*>(&s[row][col]) =
                out ? zero4() : scale4(mul, cols(c0 + col));
        __syncthreads();
        for (int q = wave; q < kPackCols / 16; q += 4) {
            const int f = c0 / 16 + q;
            if (f < nfrag) {
                f32x8 v;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = s[lane & 31][16 * q + 8 * half + j];
                const Operand<E> p = split<E>(v);
#pragma unroll
                for (int part = 0; part < kParts; ++part)
                    form[(part * nfrag + f) * 64 + lane] = p.p[part];
            }
            const int db = c0 / 32 + (q >> 1), t = q & 1;
            if (forms == 2 && db < nd) {
                f32x8 v;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = 16 * t + tile_row(j, half);
                    v[j] = s[r][32 * (q >> 1) + (lane & 31)];
                    if constexpr (kHalfT) v[j] *= half_mul;
                }
                const Operand<E> p = second_split<E, kHalfT>(v);
#pragma unroll
                for (int part = 0; part < kParts; ++part)
                    form[((kParts + part) * nfrag + t * nd + db) * 64 + lane] = p.p[part];
            }
        }
        __syncthreads();
    }
}

// Waves per SIMD, waves of a workgroup and tiles of X per wave, as the registers of
// X, the sums and a tile allow.
template <typename E, int ND, bool GRAD, bool ANSWER = false>
struct Shape {
    static constexpr bool kTwo = sizeof(E) == 4;  // fp32: two parts
    // answers hold more beside a tile: at four blocks two tiles of X and four waves per SIMD do
    // not fit (4096 x 1e6 x 128: 1427 us with one tile, 1496 with two and registers in
    // memory, 1845 with two and three waves).  At three blocks two, with 12 bytes in memory, are
    // as fast or faster (4096 x 1e6 x 96: log probabilities alone 978 us and 992, with a bias and
    // ten best 1376 and 1400)
    static constexpr int kXB = !GRAD && !kTwo && ND <= (ANSWER ? 3 : 4) ? 2 : 1;
    static constexpr int loss_occ() {
        if (kTwo) return ND <= 4 ? 4 : ND <= 8 ? 2 : 1;
        return ND <= 8 ? 4 : ND <= 12 ? 3 : 2;
    }
    static constexpr int grad_occ() {
        if (kTwo) return ND <= 1 ? 4 : ND <= 2 ? 3 : ND <= 4 ? 2 : 1;
        return ND <= 2 ? 4 : ND <= 4 ? 3 : ND <= 8 ? 2 : 1;
    }
    static constexpr int kOcc = GRAD ? grad_occ() : loss_occ();
    static constexpr int kWaves = kOcc == 4 ? 8 : 4 * kOcc;
    // Rows of up to this many blocks go through LDS whole: two records, X, the sums
    // and a tile within a wave's 512 registers.
    static constexpr int kMostStaged = !GRAD ? 16 : 12;
    static constexpr bool kStaged = ND <= kMostStaged;
    // ... one record, brought in halves, where two do not fit
    static constexpr bool kHalves = GRAD && kTwo && ND > 8;
};

// ---------------------------------------------------------------------------
// What the two kernels share: X in registers, Y's records through LDS
// ---------------------------------------------------------------------------
struct PassArgs {
    const uint8_t* x;      // records of X and of Y
    const uint8_t* y;
    int64_t x_tiles, y_tiles;
    int64_t per;           // Y tiles of a split
    int32_t x_blocks;      // workgroups along X: the first x_whole take all of Y, the
    int32_t x_whole;       // others a split of it each
    int32_t splits;
    int32_t x_groups;      // waves of a workgroup side by side along X; the others share Y
    int32_t stage;         // Y tiles of an LDS buffer
    int32_t nfrag, kd;
    int32_t forms;
    const bf16_t* x_direct;  // answers: the rows unpacked, instead of x
    int64_t x_ld, x_count;
    const bf16_t* y_rows;  // loss: the classes unpacked, instead of y
    int64_t ld, classes;
    bool first;            // the first piece of the classes: partial results are written
    // partial results of the rows behind those of the whole workgroups, one slot per
    // split and wave along Y: [slot][part_rows]...
    int64_t part_first, part_rows;
    float2* lse_part;      // loss: maximum and sum
    float4* stat_part;     // answers: top, sum and first moment, and the largest logit
    float* best;           // answers: each tile's largest logit [y tile][best_ld], or null
    int64_t best_ld;
    float* part;           // gradient: [dp], or null: to `out`
    float* bias_part;      // gradient of the bias (X: classes)
    void* out;             // x_rows x dim
    float* bias_out;
    int64_t class0;        // first class of the piece
    int64_t x_rows;
    int32_t dp, dim;
    float scale;
    bool want_bias, out_vec;
    // host: workgroups and bytes of LDS
    int64_t grid;
    int32_t lds;
};

// The workgroup's place.  Workgroups go to the eight XCDs in turn; each XCD takes a
// run of the places in the order of the splits, so that workgroups which read the
// same Y records share an L2.
struct Place {
    int32_t x_block, split;
    bool whole, none;
};
__device__ __forceinline__ Place place(const PassArgs& a, int32_t b) {
    const int32_t head = (a.x_whole + 7) / 8 * 8;
    const bool whole = b < head;
    if (!whole) b -= head;
    const int32_t wide = whole ? a.x_whole : a.x_blocks - a.x_whole;
    const int32_t total = whole ? wide : wide * a.splits, run = (total + 7) / 8;
    const int32_t k = (b & 7) * run + (b >> 3);
    return {whole ? k : a.x_whole + k % wide, whole ? 0 : k / wide, whole, k >= total};
}
inline int64_t place_grid(int64_t x_blocks, int64_t x_whole, int64_t splits) {
    return (x_whole + 7) / 8 * 8 + ((x_blocks - x_whole) * splits + 7) / 8 * 8;
}

// Copies n KB to LDS, a wave 1 KB at a time.
template <int WAVES>
__device__ __forceinline__ void copy_to_lds(const uint8_t* from, uint8_t* to, int n, int wave,
                                            int lane) {
    for (int k = wave; k < n; k += WAVES)
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void*)(from + (int64_t)k * 1024 + lane * 16),
            (__attribute__((address_space(3))) void*)(to + k * 1024), 16, 0, 0);
}

// Copies the rows of n tiles to LDS as records without a header, straight from a
// bf16 matrix of `nfrag` operands a row: each lane of an operand fetches its own 16
// bytes.  A wave takes four operands of a tile, 128 bytes of every row.
template <int WAVES>
__device__ __forceinline__ void gather_to_lds(const bf16_t* m, int64_t ld, int64_t rows,
                                              int64_t tile, uint8_t* to, int n, int nfrag,
                                              int wave, int lane) {
    const int quads = nfrag / 2 > 1 ? nfrag / 4 + (nfrag % 4 != 0) : 1;
    for (int k = wave; k < n * quads; k += WAVES) {
        const int t = k / quads, f0 = k % quads * 4;
        int64_t row = (tile + t) * 32 + (lane & 31);
        row = row < rows ? row : rows - 1;
        const bf16_t* from = m + row * ld + 16 * f0 + 8 * (lane >> 5);
#pragma unroll
        for (int f = 0; f < 4; ++f)
            if (f0 + f < nfrag)
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void*)(from + 16 * f),
                    (__attribute__((address_space(3))) void*)(to + (t * nfrag + f0 + f) * 1024),
                    16, 0, 0);
    }
}

// Waits for this wave's copies to LDS, then for all waves: what they copied has
// arrived.  A barrier by itself waits for them only where the compiler sees a read of
// theirs behind it.
__device__ __forceinline__ void copies_arrived() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Calls body(record) for this wave's Y tiles of the split: tiles yg, yg + yw, ... of
// each stage.  copy(tile, buffer, n) brings n of them to LDS.
template <int WAVES, bool STAGED, typename Copy, typename Body>
__device__ __forceinline__ void stream_records(const PassArgs& a, const Place& at_, int yg, int yw,
                                               int rec_bytes, uint8_t* lds, Copy copy, Body body) {
    const int64_t y0 = (int64_t)at_.split * a.per;
    const int64_t y1 = !at_.whole && y0 + a.per < a.y_tiles ? y0 + a.per : a.y_tiles;
    if constexpr (!STAGED) {
        for (int64_t yt = y0 + yg; yt < y1; yt += yw) body(a.y + yt * rec_bytes, yt);
    } else {
        auto tiles = [&](int64_t at) { return (int)(y1 - at < a.stage ? y1 - at : a.stage); };
        uint8_t* buf = lds;
        uint8_t* next = lds + a.stage * rec_bytes;
        if (y0 < y1) copy(y0, buf, tiles(y0));
        copies_arrived();
        for (int64_t at = y0; at < y1; at += a.stage) {
            const int64_t after = at + a.stage;
            if (after < y1) copy(after, next, tiles(after));
            const int n = tiles(at);
            for (int t = yg; t < n; t += yw) body(buf + t * rec_bytes, at + t);
            copies_arrived();
            uint8_t* b = buf;
            buf = next;
            next = b;
        }
    }
}

// The same where LDS has room for one record: it is brought in halves.  The T form of
// a tile comes while S is formed, the header and the R form of the next one while the
// second product runs; between() stands between the two, after the last read of the
// header, and every wave calls it for every tile.
// fp32 gradients, 3001 x 50021 x 384: 1526 us, 302 TFLOP/s; without LDS 6547.
template <int WAVES, typename Copy, typename Body>
__device__ __forceinline__ void stream_halves(const PassArgs& a, const Place& at_, int first_kb,
                                              int kb, uint8_t* lds, Copy copy, Body body) {
    const int64_t y0 = (int64_t)at_.split * a.per;
    const int64_t y1 = !at_.whole && y0 + a.per < a.y_tiles ? y0 + a.per : a.y_tiles;
    if (y0 < y1) copy(y0, 0, first_kb);
    for (int64_t yt = y0; yt < y1; ++yt) {
        copies_arrived();
        copy(yt, first_kb, kb);
        body(lds, yt, [&] {
            copies_arrived();
            if (yt + 1 < y1) copy(yt + 1, 0, first_kb);
        });
    }
}

// Operands of a form that a wave reads ahead of the products that use them.  An LDS
// read takes as long as two to four products; left alone the compiler reads one or
// two ahead.  DEEP: there are registers for twice as many (fp32 gradients of 160 to 256
// columns, one wave per SIMD: 1074 -> 1048 us for 3001 x 50021 x 256).
template <typename E, int N, bool DEEP = false>
struct Ahead {
    static constexpr int kMost = (DEEP ? 8 : 4) / Kind<E>::kParts;
    static constexpr int kCount = N < kMost ? N : kMost;
    Operand<E> q[kCount];

    template <typename Load>
    __device__ __forceinline__ void start(Load load) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) q[i] = load(i);
    }
    // use(i, operand i) for all of them, each read kCount uses before.
    template <int PRODUCTS, typename Load, typename Use>
    __device__ __forceinline__ void run(Load load, Use use) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            use(i, q[i % kCount]);
            if (i + kCount < N) q[i % kCount] = load(i + kCount);
        }
        constexpr int kMfma = 0x8, kDsRead = 0x100;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMfma, PRODUCTS, 0);
            if (i + kCount < N)
                __builtin_amdgcn_sched_group_barrier(kDsRead, Kind<E>::kParts, 0);
        }
    }
};

template <typename E>
constexpr int kProducts = Kind<E>::kParts == 2 ? 3 : 1;  // matrix products of two operands

// The logits of a tile against XB tiles of X, before the scales of fp32 rows.
template <typename E, int ND, int XB, bool STAGED>
__device__ __forceinline__ void tile_products(const uint8_t* rec, const Operand<E> (*x)[2 * ND],
                                              const uint8_t* const* xrec, int nfrag, int kd,
                                              int lane, f32x16* c) {
    const uint8_t* form = rec + kHeader;
    if constexpr (STAGED) {
        auto load = [&](int k) { return load_operand<E>(form, k, 2 * ND, lane); };
        Ahead<E, 2 * ND, Kind<E>::kScaled && (ND > 4)> y;
        y.start(load);
        __builtin_amdgcn_sched_barrier(0);
        y.template run<kProducts<E> * XB>(load, [&](int k, const Operand<E>& q) {
#pragma unroll
            for (int b = 0; b < XB; ++b) c[b] = product<E>(q, x[b][k], c[b]);
        });
    } else {
        for (int k = 0; k < kd; ++k) {
            const Operand<E> y = load_operand<E>(form, k, nfrag, lane);
#pragma unroll
            for (int b = 0; b < XB; ++b)
                c[b] = product<E>(y, load_operand<E>(xrec[b] + kHeader, k, nfrag, lane), c[b]);
        }
    }
}

// X's tiles of a wave.
template <int XB>
struct XTiles {
    int64_t t[XB];
    bool in[XB];  // tiles past the end repeat the last one, and are not stored
    const uint8_t* rec[XB];
};
template <int XB>
__device__ __forceinline__ XTiles<XB> x_tiles_of(const PassArgs& a, int x_block, int xg,
                                                 int rec_bytes) {
    XTiles<XB> r;
#pragma unroll
    for (int b = 0; b < XB; ++b) {
        int64_t t = ((int64_t)x_block * a.x_groups + xg) * XB + b;
        r.in[b] = t < a.x_tiles;
        if (!r.in[b]) t = a.x_tiles - 1;
        r.t[b] = t;
        r.rec[b] = a.x + t * rec_bytes;
    }
    return r;
}

// ---------------------------------------------------------------------------
// Loss: running maximum and sum
// ---------------------------------------------------------------------------
// exp(a - b) for a <= b, 0 where a is -inf (also if b is).
__device__ __forceinline__ float exp_below(float a, float b) {
    return a == -INFINITY ? 0.f : exp2f((a - b) * kLog2e);
}

constexpr float kRise = 8.f;

// What a row's classes leave: with e = exp2(u), u = (x - top) log2(e), the sum of e and,
// for the entropy log sum - ln(2) first / sum, that of u e.  `top` need not be the
// maximum: a rise by a few is a few more bits of u in `first`, so that answers allow less.
struct Stats {
    float top, sum, first;
};
constexpr float kRiseAnswer = 2.f;

// The same from another top at or above.
__device__ __forceinline__ Stats raise(Stats s, float top) {
    const float d = (s.top - top) * kLog2e, f = __builtin_amdgcn_exp2f(d);
    return {top, s.sum * f, f * fmaf(d, s.sum, s.first)};
}
__device__ __forceinline__ Stats join(Stats a, Stats b) {
    const float top = fmaxf(a.top, b.top);
    a = raise(a, top), b = raise(b, top);
    return {top, a.sum + b.sum, a.first + b.first};
}

// Bound by the vector units, which take the exponential, its argument and the sum of
// every element: 4096 x 1e6 x 128 bf16 from records 960 to 1040 us (1.0 PFLOP/s; 72%
// of the time a SIMD issues vector instructions, 52% its matrix core works), by the
// clock, which falls under it.  3001 x 50021 x 256 fp32: 194 to 204 us, 377 to 396
// TFLOP/s.
template <typename E, int ND, int XB, int WAVES, int OCC, bool STAGED, bool DIRECT, bool ANSWER>
__global__ __launch_bounds__(WAVES * 64) __attribute__((amdgpu_waves_per_eu(OCC, OCC)))
void k_sm_lse(PassArgs a) {
    extern __shared__ __align__(16) uint8_t lds[];
    const Place at = place(a, blockIdx.x);
    if (at.none) return;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int xg = wave % a.x_groups, yg = wave / a.x_groups, yw = WAVES / a.x_groups;
    const int nfrag = STAGED ? 2 * ND : a.nfrag;
    const int rec_bytes = record_bytes(nfrag, Kind<E>::kParts, a.forms);
    const XTiles<XB> xt = x_tiles_of<XB>(a, at.x_block, xg, rec_bytes);
    Operand<E> x[XB][2 * ND];
    // the first moment in a few running sums, so that each takes one addition in so many
    constexpr int kSums = Kind<E>::kScaled ? 2 : 4;
    float xmul[XB], top[XB], sum[XB], first[XB][kSums], most[XB];
#pragma unroll
    for (int b = 0; b < XB; ++b) {
        if constexpr (STAGED) {
            bool packed = true;
            if constexpr (ANSWER && !Kind<E>::kScaled) {
                packed = a.x_direct == nullptr;
                if (!packed) {
                    // whole operands: 16 bytes of the lane's row each
                    const int64_t row = xt.t[b] * 32 + (lane & 31);
                    const bf16_t* from = a.x_direct + (row < a.x_count ? row : a.x_count - 1) * a.x_ld;
#pragma unroll
                    for (int k = 0; k < 2 * ND; ++k)
                        x[b][k].p[0] = *reinterpret_cast<const typename Kind<E>::Vec*>(
                            from + 16 * k + 8 * half);
                }
            }
            if (packed) {
#pragma unroll
                for (int k = 0; k < 2 * ND; ++k)
                    x[b][k] = load_operand<E>(xt.rec[b] + kHeader, k, 2 * ND, lane);
            }
        }
        xmul[b] = Kind<E>::kScaled ? field(xt.rec[b], kMul)[lane & 31] : 1.f;
        top[b] = ANSWER ? kLeast : -INFINITY;
        sum[b] = 0.f;
#pragma unroll
        for (int k = 0; k < kSums; ++k) first[b][k] = 0.f;
        most[b] = kFloor;
    }
    // DIRECT: no headers; there is no bias then, only the end of the classes
    const int y_bytes = DIRECT ? 2 * ND * 1024 : rec_bytes;
    stream_records<WAVES, STAGED>(
        a, at, yg, yw, y_bytes, lds,
        [&](int64_t tile, uint8_t* to, int n) {
            if constexpr (DIRECT)
                gather_to_lds<WAVES>(a.y_rows, a.ld, a.classes, tile, to, n, 2 * ND, wave, lane);
            else
                copy_to_lds<WAVES>(a.y + tile * rec_bytes, to, n * (rec_bytes / 1024), wave, lane);
        },
        [&](const uint8_t* rec, int64_t yt) {
            f32x16 c[XB], term = {};
            if constexpr (!DIRECT) {
                term = row_values(rec, kTerm, half);
            } else if (!ANSWER && yt * 32 + 32 > a.classes) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (yt * 32 + tile_row(i, half) >= a.classes) term[i] = -INFINITY;
            }
#pragma unroll
            for (int b = 0; b < XB; ++b) c[b] = Kind<E>::kScaled ? f32x16{} : term;
            tile_products<E, ND, XB, STAGED>(DIRECT ? rec - kHeader : rec, x, xt.rec, nfrag, a.kd,
                                             lane, c);
            if constexpr (Kind<E>::kScaled) {
                const f32x16 ymul = row_values(rec, kMul, half);
#pragma unroll
                for (int b = 0; b < XB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        c[b][i] = fmaf(c[b][i] * ymul[i], xmul[b], term[i]);
            }
            // behind the products: their sum then starts from a constant 0, which costs nothing,
            // and not from 16 registers that are filled for every tile
            if constexpr (ANSWER && DIRECT) {
                if (yt * 32 + 32 > a.classes) {
#pragma unroll
                    for (int b = 0; b < XB; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (yt * 32 + tile_row(i, half) >= a.classes) c[b][i] = kFloor;
                }
            }
            // `top` is where the sums' exponentials start from, and is raised only when a
            // logit is far above it: sums of a few hundred e^kRise are no trouble
#pragma unroll
            for (int b = 0; b < XB; ++b) {
                float m = c[b][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) m = fmaxf(m, c[b][i]);
                if constexpr (ANSWER) {
                    if (a.best != nullptr) {
                        const int mi = __float_as_int(m);
                        const auto both = __builtin_amdgcn_permlane32_swap(mi, mi, false, false);
                        const float of_tile =
                            fmaxf(__int_as_float(both[0]), __int_as_float(both[1]));
                        if (half == 0 && xt.in[b])
                            a.best[yt * a.best_ld + xt.t[b] * 32 + lane] = of_tile;
                    }
                    most[b] = fmaxf(most[b], m);
                    if (__ballot(m > top[b] + kRiseAnswer) != 0) {
                        const float up = fmaxf(m, top[b]), d = (top[b] - up) * kLog2e;
                        const float f = __builtin_amdgcn_exp2f(d);
                        first[b][0] = fmaf(d, sum[b], first[b][0]);
#pragma unroll
                        for (int k = 0; k < kSums; ++k) first[b][k] *= f;
                        sum[b] *= f;
                        top[b] = up;
                    }
                    const float sub = -top[b] * kLog2e;
                    // in two halves, so that few of the logarithms are held at a time
#pragma unroll
                    for (int j = 0; j < 16; j += 8) {
                        float s[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float u = fmaf(c[b][j + i], kLog2e, sub);
                            const float v = fmaf(c[b][j + 4 + i], kLog2e, sub);
                            const float e = __builtin_amdgcn_exp2f(u), g = __builtin_amdgcn_exp2f(v);
                            s[i] = e + g;
                            float& of_sum = first[b][i % kSums];
                            of_sum = fmaf(v, g, fmaf(u, e, of_sum));
                        }
                        sum[b] += (s[0] + s[1]) + (s[2] + s[3]);
                    }
                } else {
                    if (__ballot(m > top[b] + kRise) != 0) {
                        const float up = fmaxf(m, top[b]);
                        sum[b] *= exp_below(top[b], up);
                        top[b] = up;
                    }
                    const float sub = top[b] == -INFINITY ? 0.f : -top[b] * kLog2e;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        c[b][i] = __builtin_amdgcn_exp2f(fmaf(c[b][i], kLog2e, sub));
                    sum[b] += sum16(c[b]);
                }
            }
        });
    if constexpr (ANSWER) {
#pragma unroll
        for (int b = 0; b < XB; ++b) {
            // the halves hold different classes of the same row
            float of_lane = first[b][0] + first[b][1];
            if constexpr (kSums == 4) of_lane += first[b][2] + first[b][3];
            Stats s = join({top[b], sum[b], of_lane},
                           {__shfl_xor(top[b], 32), __shfl_xor(sum[b], 32), __shfl_xor(of_lane, 32)});
            float largest = fmaxf(most[b], __shfl_xor(most[b], 32));
            if (half == 0 && xt.in[b]) {
                float4* out = a.stat_part + ((int64_t)at.split * yw + yg) * a.part_rows +
                              xt.t[b] * 32 + lane;
                if (!a.first) {
                    const float4 p = *out;
                    s = join(s, {p.x, p.y, p.z});
                    largest = fmaxf(largest, p.w);
                }
                *out = make_float4(s.top, s.sum, s.first, largest);
            }
        }
        return;
    }
#pragma unroll
    for (int b = 0; b < XB; ++b) {
        // the halves hold different classes of the same row
        const float top2 = __shfl_xor(top[b], 32), sum2 = __shfl_xor(sum[b], 32);
        float m = fmaxf(top[b], top2);
        float v = sum[b] * exp_below(top[b], m) + sum2 * exp_below(top2, m);
        if (half == 0 && xt.in[b]) {
            float2* out = a.lse_part + ((int64_t)at.split * yw + yg) * a.part_rows +
                          xt.t[b] * 32 + lane;
            if (!a.first) {
                const float2 p = *out;
                const float mm = fmaxf(m, p.x);
                v = v * exp_below(m, mm) + p.y * exp_below(p.x, mm);
                m = mm;
            }
            *out = make_float2(m, v);
        }
    }
}

// ---------------------------------------------------------------------------
// Loss of few rows
// ---------------------------------------------------------------------------
// With few rows the table is read once and that is all: no packing.  A wave takes
// 16 classes at a time, each lane 16 bytes of one class's row, which are an operand
// of a 16x16 product as they lie (fp32: exact fp32 products); the rows h are the
// other operand, from LDS.  A lane then holds four classes' logits of one row.
// Loads run one group of kFewGroup operands ahead.  One row is bound by memory: 1e6 x
// 128 fp32 take 87 us of the kernel, 5.9 TB/s; up to 16 rows' whole call 100 us (bf16
// 54), 64 rows of bf16 67.  From 33 rows up the exact fp32
// products bind, 64 x 300000 x 256 at 69 TFLOP/s with the host's work.
//
// h takes LDS, up to kFewLds, and so leaves a CU one workgroup where it is wide: four
// waves of 16 rows each have to themselves, more rows get eight (38 rows, 762366 x
// 336 fp32: 403 us against 581 with four, one row: 106 against 104).  fp32 rows that
// do not fit go through the packed records, whose traffic is three times the table
// (the same call: 772 us); bf16 rows do above 60 KB, where their packing costs less
// than the one workgroup (64 rows, 300000 x 512: 88 us against 96).
constexpr int kFewGroup = 8;
constexpr int few_waves(int nb) { return nb == 1 ? 4 : 8; }
template <typename E>
constexpr int kFewLds = (sizeof(E) == 2 ? 60 : 144) * 1024;

typedef float f32x4v __attribute__((ext_vector_type(4)));

template <typename E>
struct Few;
template <>
struct Few<bf16_t> {
    static constexpr int kCols = 32;   // columns of a 16x16 product
    using Vec = bf16x8;
    static __device__ __forceinline__ f32x4v mfma(Vec a, Vec b, f32x4v c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Few<float> {
    static constexpr int kCols = 16;   // of four 16x16x4 products
    using Vec = f32x4;
    static __device__ __forceinline__ f32x4v mfma(Vec a, Vec b, f32x4v c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// Operands of a row; of codes and of thirds whole pairs.
template <typename E, bool CODES, bool THIRDS = false>
__host__ __device__ constexpr int few_operands(int dim) {
    return CODES ? 2 * ((dim + 63) / 64)
                 : THIRDS ? 2 * ((dim + 31) / 32) : (dim + Few<E>::kCols - 1) / Few<E>::kCols;
}
// KB of LDS for a block of 16 rows.
template <typename E, bool CODES, bool THIRDS = false>
__host__ __device__ constexpr int few_kb(int dim) {
    return THIRDS ? 3 * ((dim + 31) / 32) : few_operands<E, CODES>(dim);
}

// 16 bytes of a row at a column, 0 past its end, read BYTES at a time.
template <typename E, int BYTES>
__device__ __forceinline__ typename Few<E>::Vec load_few_cols(const E* row, int col, int dim) {
    using Vec = typename Few<E>::Vec;
    constexpr int kN = 16 / sizeof(E);
    union {
        Vec v;
        E e[kN];
    } u;
    if constexpr (BYTES == 16) {
        u.v = col < dim ? *reinterpret_cast<const Vec*>(row + col) : Vec{};
    } else if constexpr (BYTES == 8) {  // bf16 rows of an odd number of fours
        typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
        const u16x4 a = col < dim ? *reinterpret_cast<const u16x4*>(row + col) : u16x4{};
        const u16x4 b = col + 4 < dim ? *reinterpret_cast<const u16x4*>(row + col + 4) : u16x4{};
#pragma unroll
        for (int j = 0; j < 4; ++j) u.e[j] = a[j], u.e[4 + j] = b[j];
    } else {
#pragma unroll
        for (int j = 0; j < kN; ++j) u.e[j] = col + j < dim ? row[col + j] : (E)0;
    }
    return u.v;
}

// The classes' rows as a wave of k_sm_few reads them: a group of GROUP operands in
// flight, then one operand at a time.
template <typename E, int BYTES, bool CODES, int GROUP>
struct FewTable {
    using F = Few<E>;
    using Vec = typename F::Vec;
    static constexpr int kN = 16 / sizeof(E);
    Vec v[GROUP];

    // First column of operand k in lane quad q.
    static __device__ __forceinline__ int column(int k, int q) { return F::kCols * k + kN * q; }
    __device__ __forceinline__ void fetch(const SoftmaxArgs& a, int64_t row, int g, int ops, int quad) {
        const E* w = static_cast<const E*>(a.w) + row * a.ld_w;
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            if (g * GROUP + i < ops)
                v[i] = load_few_cols<E, BYTES>(w, column(g * GROUP + i, quad), a.dim);
    }
    __device__ __forceinline__ Vec operand(int i) const { return v[i]; }
};

// A table in 8 bits: a lane takes 16 codes at a time, which are two operands of a bf16
// product (whose columns are taken in that order), and their scale.
template <int BYTES, int GROUP>
struct FewTable<bf16_t, BYTES, true, GROUP> {
    using Vec = bf16x8;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    u32x4 q[GROUP / 2];
    uint32_t scale[GROUP / 2];

    static __device__ __forceinline__ int column(int k, int q) {
        return 64 * (k >> 1) + 16 * q + 8 * (k & 1);
    }
    __device__ __forceinline__ void fetch(const SoftmaxArgs& a, int64_t row, int g, int ops, int quad) {
        const uint8_t* w = static_cast<const uint8_t*>(a.w) + row * a.ld_w;
        const uint8_t* s = a.w_scales + row * a.ld_scales;
#pragma unroll
        for (int i = 0; i < GROUP; i += 2) {
            const int col = column(g * GROUP + i, quad);
            u32x4 r = {};
            uint32_t b = 127;
            if (col < a.dim) {
                b = s[col / kByteBlock];
                if constexpr (BYTES == 16) {
                    r = *reinterpret_cast<const u32x4*>(w + col);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int c = col + 4 * j;
                        if (c >= a.dim) continue;
                        if constexpr (BYTES == 4) r[j] = *reinterpret_cast<const uint32_t*>(w + c);
                        else r[j] = w[c] | w[c + 1] << 8 | w[c + 2] << 16 | (uint32_t)w[c + 3] << 24;
                    }
                }
            }
            q[i / 2] = r;
            scale[i / 2] = b;
        }
    }
    __device__ __forceinline__ Vec operand(int i) const {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const float mul = byte_scale(scale[i / 2]);
        Vec v;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t w = q[i / 2][2 * (i & 1) + j];
            const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, mul, false);
            const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, mul, true);
            v[4 * j] = lo[0], v[4 * j + 1] = lo[1], v[4 * j + 2] = hi[0], v[4 * j + 3] = hi[1];
        }
        return v;
    }
};

// The largest over the four lanes that are 16 apart (as xor_add).
__device__ __forceinline__ float quads_max(float v) {
    const int a = __float_as_int(v);
    const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    v = fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
    const int b = __float_as_int(v);
    const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return fmaxf(__int_as_float(q[0]), __int_as_float(q[1]));
}

// An fp32 number as the sum of three bf16 ones, each the nearest to what the ones before
// leave: within 2^-27 of it.  Of the nine products of two such sums the six above 2^-27 are
// formed, the smallest first, which is an fp32 product but for its rounding, at six bf16
// products in place of eight fp32 ones of twice the time each.
struct Thirds {
    bf16x8 p[3];
};
__device__ __forceinline__ Thirds thirds(f32x4 a, f32x4 b) {
    f32x8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    Thirds r;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        r.p[k] = __builtin_convertvector(v, bf16x8);
        v -= __builtin_convertvector(r.p[k], f32x8);
    }
    return r;
}

// NB blocks of 16 rows.  Of a table in 8 bits the operands come in pairs.  THIRDS: so do
// those of fp32 rows, each pair of 16 columns as one of 32 in three parts.
template <typename E, int NB, int BYTES, bool ANSWER, bool CODES, bool THIRDS>
__global__ __launch_bounds__(few_waves(NB) * 64, THIRDS ? 4 : 1) void k_sm_few(SoftmaxArgs a, int64_t tiles,
                                                               void* __restrict__ parts,
                                                               int64_t pad, int64_t slots,
                                                               int64_t slot0,
                                                               float* __restrict__ best) {
    constexpr int kWaves = few_waves(NB);
    using F = Few<E>;
    using Vec = typename F::Vec;
    // thirds need the registers of half a group
    constexpr int kGroup = THIRDS ? kFewGroup / 2 : kFewGroup;
    using Table = FewTable<E, BYTES, CODES, kGroup>;
    using Part = std::conditional_t<ANSWER, float4, float2>;
    Part* part = static_cast<Part*>(parts);
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ Part s_part[kWaves][NB * 16];
    Vec* sh = reinterpret_cast<Vec*>(lds);  // [operand][block of rows][lane]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quad = lane >> 4;
    const int ops = few_operands<E, CODES, THIRDS>(a.dim);
    // h's alignment is its own where the table is in 8 bits
    constexpr int kBytesH = CODES ? 2 : BYTES;
    bf16x8* sh3 = reinterpret_cast<bf16x8*>(lds);  // [pair][part][block of rows][lane]
    for (int j = threadIdx.x; j < (THIRDS ? ops / 2 : ops) * NB * 64; j += kWaves * 64) {
        const int l = j & 63, b = (j >> 6) % NB, k = (j >> 6) / NB;
        const int64_t row = 16 * b + (l & 15);
        if constexpr (THIRDS) {
            f32x4 v[2] = {};
            if (row < a.n) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    v[e] = load_few_cols<E, kBytesH>(static_cast<const E*>(a.h) + row * a.ld_h,
                                                     Table::column(2 * k + e, l >> 4), a.dim);
            }
            const Thirds r = thirds(v[0], v[1]);
#pragma unroll
            for (int part = 0; part < 3; ++part) sh3[((k * 3 + part) * NB + b) * 64 + l] = r.p[part];
            continue;
        }
        sh[j] = row < a.n ? load_few_cols<E, kBytesH>(static_cast<const E*>(a.h) + row * a.ld_h,
                                                    Table::column(k, l >> 4), a.dim)
                          : Vec{};
    }
    __syncthreads();
    const int groups = (ops + kGroup - 1) / kGroup;
    const int64_t step = (int64_t)gridDim.x * kWaves;
    int64_t tile = (int64_t)blockIdx.x * kWaves + wave;
    auto fetch = [&](int64_t t, int g, Table& v) {
        int64_t row = t * 16 + (lane & 15);
        row = row < a.classes ? row : a.classes - 1;
        v.fetch(a, row, g, ops, quad);
    };
    float top[NB], sum[NB], first[NB];
    f32x4v c[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        top[b] = ANSWER ? kLeast : -INFINITY;
        sum[b] = 0.f;
        first[b] = 0.f;
        c[b] = f32x4v{};
    }
    Table now, next;
    if (tile < tiles) fetch(tile, 0, now);
    int g = 0;
    while (tile < tiles) {
        const bool last = g + 1 == groups;
        const int64_t next_tile = last ? tile + step : tile;
        if (next_tile < tiles) fetch(next_tile, last ? 0 : g + 1, next);
        float term[4];
        if (last) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t k = tile * 16 + 4 * quad + i;
                term[i] = k >= a.classes ? -INFINITY : a.bias == nullptr ? 0.f : a.bias[k];
            }
        }
        if constexpr (THIRDS) {
#pragma unroll
            for (int i = 0; i < kGroup; i += 2)
                if (g * kGroup + i < ops) {
                    const Thirds w = thirds(now.operand(i), now.operand(i + 1));
                    const int pair = (g * kGroup + i) / 2;
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        bf16x8 h[3];
#pragma unroll
                        for (int part = 0; part < 3; ++part)
                            h[part] = sh3[((pair * 3 + part) * NB + b) * 64 + lane];
                        using B = Few<bf16_t>;
                        c[b] = B::mfma(w.p[2], h[0], c[b]);
                        c[b] = B::mfma(w.p[0], h[2], c[b]);
                        c[b] = B::mfma(w.p[1], h[1], c[b]);
                        c[b] = B::mfma(w.p[1], h[0], c[b]);
                        c[b] = B::mfma(w.p[0], h[1], c[b]);
                        c[b] = B::mfma(w.p[0], h[0], c[b]);
                    }
                }
        } else
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
            if (g * kGroup + i < ops) {
                const Vec w = now.operand(i);
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    c[b] = F::mfma(w, sh[((g * kGroup + i) * NB + b) * 64 + lane], c[b]);
            }
        if (last) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if constexpr (ANSWER) {
                    float x[4], m = kFloor;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[i] = term[i] < kLeast ? kFloor : c[b][i] + term[i];
                        m = fmaxf(m, x[i]);
                    }
                    if (best != nullptr) {
                        const float t = quads_max(m);
                        if (lane < 16) best[tile * pad + 16 * b + lane] = t;
                    }
                    if (__ballot(m > top[b]) != 0) {
                        const Stats s = raise({top[b], sum[b], first[b]}, fmaxf(m, top[b]));
                        top[b] = s.top, sum[b] = s.sum, first[b] = s.first;
                    }
                    const float sub = -top[b] * kLog2e;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float u = fmaf(x[i], kLog2e, sub), e = __builtin_amdgcn_exp2f(u);
                        sum[b] += e;
                        first[b] = fmaf(u, e, first[b]);
                    }
                } else {
                    float x[4], m = top[b];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // a class that is out counts for nothing, whatever its row holds
                        x[i] = term[i] == -INFINITY ? -INFINITY : c[b][i] + term[i];
                        m = fmaxf(m, x[i]);
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
                    sum[b] *= exp_below(top[b], ref);
                    top[b] = m;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sum[b] += __builtin_amdgcn_exp2f(fmaf(x[i], kLog2e, -ref * kLog2e));
                }
                c[b] = f32x4v{};
            }
        }
        now = next;
        tile = next_tile;
        g = last ? 0 : g + 1;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        if constexpr (ANSWER) {
            Stats s{top[b], sum[b], first[b]};
#pragma unroll
            for (int off = 16; off < 64; off <<= 1)
                s = join(s, {__shfl_xor(s.top, off), __shfl_xor(s.sum, off),
                             __shfl_xor(s.first, off)});
            // the top of few rows is the maximum
            if (lane < 16) s_part[wave][16 * b + lane] = make_float4(s.top, s.sum, s.first, s.top);
        } else {
#pragma unroll
            for (int off = 16; off < 64; off <<= 1) {
                const float t2 = __shfl_xor(top[b], off), s2 = __shfl_xor(sum[b], off);
                const float m = fmaxf(top[b], t2);
                sum[b] = sum[b] * exp_below(top[b], m) + s2 * exp_below(t2, m);
                top[b] = m;
            }
            if (lane < 16) s_part[wave][16 * b + lane] = make_float2(top[b], sum[b]);
        }
    }
    __syncthreads();
    if (threadIdx.x < NB * 16) {
        Part r = s_part[0][threadIdx.x];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) {
            const Part q = s_part[k][threadIdx.x];
            if constexpr (ANSWER) {
                const Stats s = join({r.x, r.y, r.z}, {q.x, q.y, q.z});
                r = make_float4(s.top, s.sum, s.first, s.top);
            } else {
                const float m = fmaxf(r.x, q.x);
                r.y = r.y * exp_below(r.x, m) + q.y * exp_below(q.x, m);
                r.x = m;
            }
        }
            // of answers a row's entries are adjacent, which few threads then join
        part[ANSWER ? threadIdx.x * slots + slot0 + blockIdx.x : blockIdx.x * pad + threadIdx.x] = r;
    }
}

// ---------------------------------------------------------------------------
// Gradients
// ---------------------------------------------------------------------------
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

// Four elements of a result; vec: the array is aligned for four (its element type is
// all that the caller owes).
template <typename E>
__device__ __forceinline__ void store_out(E* p, float4 v, float scale, bool vec) {
    const f32x4 q = {v.x * scale, v.y * scale, v.z * scale, v.w * scale};
    if constexpr (sizeof(E) == 4) {
        if (vec) {
            *reinterpret_cast<f32x4*>(p) = q;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = q[e];
        }
    } else {
        const u16x4 u = __builtin_bit_cast(u16x4, __builtin_convertvector(q, bf16x4));
        if (vec) {
            *reinterpret_cast<u16x4*>(p) = u;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = u[e];
        }
    }
}

// ROWS: X are the rows and Y the classes (dh), else X are the classes (dw).
template <typename E, int ND, int XB, int WAVES, bool STAGED, bool ROWS, bool ANSWER>
__device__ __forceinline__ void grad_block(const PassArgs& a, int32_t block, uint8_t* lds) {
    constexpr bool kScaled = Kind<E>::kScaled;
    // bf16 rows of answers: G in halves under a scale, as fp32 rows' G, not in bf16
    constexpr bool kHalfBits = ANSWER && !kScaled;
    // one wave per SIMD
    constexpr bool kKeepsSums = STAGED && (kScaled ? ND > 4 : kHalfBits && ND > 8);
    constexpr bool HALVES = STAGED && Shape<E, ND, true>::kHalves;
    const Place at = place(a, block);
    if (at.none) return;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int xg = wave % a.x_groups, yg = wave / a.x_groups, yw = WAVES / a.x_groups;
    const int nfrag = STAGED ? 2 * ND : a.nfrag;
    const int rec_bytes = record_bytes(nfrag, Kind<E>::kParts, 2);
    const int db0 = blockIdx.y * ND, nd = nfrag / 2;
    const XTiles<XB> xt = x_tiles_of<XB>(a, at.x_block, xg, rec_bytes);
    Operand<E> x[XB][2 * ND];
    // per X row: the factor and the term of its exponents (a class's bias is the
    // initial value of its column where that is not scaled), the label (for
    // classes: the class itself) and the weight
    float xmul[XB], xterm[XB], xw[XB], bias[XB], pscale[XB], xslope[XB], xcoef[XB], xbound[XB];
    int32_t xl[XB];
    f32x16 acc[XB][ND];
#pragma unroll
    for (int b = 0; b < XB; ++b) {
        if constexpr (STAGED) {
#pragma unroll
            for (int k = 0; k < 2 * ND; ++k)
                x[b][k] = load_operand<E>(xt.rec[b] + kHeader, k, 2 * ND, lane);
        }
        const int r = lane & 31;
        xmul[b] = kScaled ? field(xt.rec[b], kMul)[r] * kLog2e : kLog2e;
        xterm[b] = field(xt.rec[b], ROWS || kScaled ? kTerm2 : kTerm)[r];
        xw[b] = ROWS ? field(xt.rec[b], kWeight)[r] : 0.f;
        xslope[b] = ROWS && ANSWER ? field(xt.rec[b], kSlope)[r] : 0.f;
        xcoef[b] = ROWS && ANSWER ? field(xt.rec[b], kCoef)[r] : 0.f;
        xbound[b] = ROWS && ANSWER ? element_bound(xslope[b], xcoef[b], xw[b]) : 0.f;
        const int32_t label = lane_label(xt.rec[b], lane);
        // classes fit 31 bits; a label of an earlier piece is below 0 here
        xl[b] = (int32_t)(ROWS ? (label < 0 ? -1 : label - a.class0)
                               : a.class0 + xt.t[b] * 32 + r);
        bias[b] = 0.f;
        pscale[b] = 0.f;  // until an element is not 0
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[b][d] = f32x16{};
    }
    auto body = [&](const uint8_t* rec, int64_t yt, auto between) {
        f32x16 c[XB];
#pragma unroll
        for (int b = 0; b < XB; ++b) {
            if constexpr (kScaled) {
                c[b] = f32x16{};
            } else if constexpr (ROWS) {
                c[b] = row_values(rec, kTerm, half);
            } else {
                // written anew for every tile: kept, it would take 16 registers
                float bias0 = xterm[b];
                asm("" : "+v"(bias0));
#pragma unroll
                for (int i = 0; i < 16; ++i) c[b][i] = bias0;
            }
        }
        tile_products<E, ND, XB, STAGED>(rec, x, xt.rec, nfrag, a.kd, lane, c);
        // the first operands of the second product are read behind the exponentials
        const uint8_t* form = rec + kHeader + Kind<E>::kParts * nfrag * 1024;
        auto load = [&](int f) {
            return load_operand<E>(form, (f / ND) * nd + db0 + f % ND, nfrag, lane);
        };
        Ahead<E, 2 * ND, STAGED && kScaled && (ND > 4)> y;
        if constexpr (!HALVES) {
            y.start(load);
            __builtin_amdgcn_sched_barrier(0);
        }
        // probabilities times the weight
        if constexpr (ANSWER) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 ymul, yterm, yslope, ycoef;
                if constexpr (kScaled) ymul = row_four(rec, kMul, half, g);
                if constexpr (kScaled || !ROWS) yterm = row_four(rec, kTerm2, half, g);
                if constexpr (!ROWS)
                    yslope = row_four(rec, kSlope, half, g), ycoef = row_four(rec, kCoef, half, g);
#pragma unroll
                for (int b = 0; b < XB; ++b)
#pragma unroll
                    for (int i = 4 * g; i < 4 * g + 4; ++i) {
                        float u;
                        if constexpr (kScaled)
                            u = fmaf(c[b][i] * ymul[i - 4 * g], xmul[b], yterm[i - 4 * g]) + xterm[b];
                        else
                            u = fmaf(c[b][i], kLog2e, ROWS ? xterm[b] : yterm[i - 4 * g]);
                        c[b][i] = __builtin_amdgcn_exp2f(u) *
                                  fmaf(u, ROWS ? xslope[b] : yslope[i - 4 * g],
                                       ROWS ? xcoef[b] : ycoef[i - 4 * g]);
                    }
            }
        } else if constexpr (kScaled) {
            const f32x16 ymul = row_values(rec, kMul, half);
            const f32x16 yterm = row_values(rec, kTerm2, half);
#pragma unroll
            for (int b = 0; b < XB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    c[b][i] = __builtin_amdgcn_exp2f(
                        fmaf(c[b][i] * ymul[i], xmul[b], yterm[i]) + xterm[b]);
        } else if constexpr (ROWS) {
#pragma unroll
            for (int b = 0; b < XB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    c[b][i] = __builtin_amdgcn_exp2f(fmaf(c[b][i], kLog2e, xterm[b]));
        } else {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 yterm = row_four(rec, kTerm2, half, g);
#pragma unroll
                for (int b = 0; b < XB; ++b)
#pragma unroll
                    for (int i = 4 * g; i < 4 * g + 4; ++i)
                        c[b][i] = __builtin_amdgcn_exp2f(fmaf(c[b][i], kLog2e, yterm[i - 4 * g]));
            }
        }
        // the labels' elements, in the tiles that hold one
#pragma unroll
        for (int b = 0; b < XB; ++b) {
            if constexpr (ROWS) {
                const int32_t d = xl[b] - (int32_t)yt * 32;
                if (__ballot((uint32_t)d < 32u) != 0) {
                    const int32_t e = d - 4 * half;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (e == tile_row(i, 0)) c[b][i] -= xw[b];
                }
            } else {
                const int32_t d = lane_label(rec, lane) - (int32_t)(a.class0 + xt.t[b] * 32);
                if (__ballot((uint32_t)d < 32u) != 0) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 label = row_four(rec, kLabel, half, g);
                        const f32x4 weight = row_four(rec, kWeight, half, g);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (__float_as_int(label[i]) == xl[b]) c[b][4 * g + i] -= weight[i];
                    }
                }
                if (a.want_bias) {
                    bias[b] += sum16(c[b]);
                }
            }
        }
        // a new scale for the sums of X's row b, whose next element is up to `big`
        auto scale_sums = [&](int b, float big, bool anew, int below) {
            // big is below 2^e: it is brought below 2^below
            float ratio = 1.f;
            if (anew) {
                const int e = __builtin_amdgcn_frexp_expf(big);
                const float s = ldexpf(1.f, e < below - 120 ? 120 : below - e);
                ratio = pscale[b] > 0.f ? fminf(s / pscale[b], 1.f) : 0.f;
                pscale[b] = pscale[b] > 0.f ? fminf(s, pscale[b]) : s;
            }
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                // a wave alone on its SIMD keeps the sums in accumulation registers; unless
                // that is said here, the compiler copies them for this product in every tile
                if constexpr (kKeepsSums) asm volatile("" : "+a"(acc[b][d]));
                acc[b][d] *= ratio;
                if constexpr (kKeepsSums) asm volatile("" : "+a"(acc[b][d]));
            }
        };
        if constexpr (kScaled) {
            const f32x16 ymul = row_values(rec, kMul, half);
#pragma unroll
            for (int b = 0; b < XB; ++b) {
                float big = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    c[b][i] *= ymul[i];
                    big = fmaxf(big, fabsf(c[b][i]));
                }
                // the halves share the sums of a row: they share its scale
                big = fmaxf(big, __shfl_xor(big, 32));
                const bool anew = big * pscale[b] > 0x1p15f || (pscale[b] == 0.f && big > 0.f);
                if (__ballot(anew) != 0) scale_sums(b, big, anew, 15);
                c[b] *= pscale[b];
            }
        } else if constexpr (kHalfBits) {
            // A row's elements are scaled by what they can be: its label's is about that large.
            // A class may have small ones alone, and is scaled by those that it has.  Either
            // way the largest is brought below 2^11 or 2^12, so that few later ones are too large
            const float record_mul = row_four(rec, kMul, 0, 0)[0];
#pragma unroll
            for (int b = 0; b < XB; ++b) {
                float big = xbound[b];
                if constexpr (!ROWS) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) big = fmaxf(big, fabsf(c[b][i]));
                    const int v = __float_as_int(big);
                    const auto both = __builtin_amdgcn_permlane32_swap(v, v, false, false);
                    big = fmaxf(__int_as_float(both[0]), __int_as_float(both[1]));
                }
                big *= record_mul;
                const bool anew = big * pscale[b] > 0x1p15f || (pscale[b] == 0.f && big > 0.f);
                if (__ballot(anew) != 0) scale_sums(b, big, anew, ROWS ? 12 : 11);
                c[b] *= record_mul * pscale[b];
            }
        }
        Operand<E> p[XB][2];
#pragma unroll
        for (int b = 0; b < XB; ++b)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x8 v;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = c[b][8 * t + j];
                p[b][t] = second_split<E, kHalfBits>(v);
            }
        if constexpr (HALVES) {
            between();
            y.start(load);
            __builtin_amdgcn_sched_barrier(0);
        }
        y.template run<kProducts<E> * XB>(load, [&](int f, const Operand<E>& q) {
#pragma unroll
            for (int b = 0; b < XB; ++b)
                acc[b][f % ND] = second_product<E, kHalfBits>(q, p[b][f / ND], acc[b][f % ND]);
        });
    };
    if constexpr (HALVES) {
        stream_halves<WAVES>(
            a, at, rec_bytes / 1024 - Kind<E>::kParts * nfrag, rec_bytes / 1024, lds,
            [&](int64_t tile, int kb0, int kb1) {
                copy_to_lds<WAVES>(a.y + tile * rec_bytes + kb0 * 1024, lds + kb0 * 1024, kb1 - kb0,
                                   wave, lane);
            },
            body);
    } else {
        stream_records<WAVES, STAGED>(
            a, at, yg, yw, rec_bytes, lds,
            [&](int64_t tile, uint8_t* to, int n) {
                copy_to_lds<WAVES>(a.y + tile * rec_bytes, to, n * (rec_bytes / 1024), wave, lane);
            },
            [&](const uint8_t* rec, int64_t yt) { body(rec, yt, [] {}); });
    }
#pragma unroll
    for (int b = 0; b < XB; ++b) {
        if (!xt.in[b]) continue;
        const int64_t xi = xt.t[b] * 32 + (lane & 31);
        const int64_t row = ((int64_t)at.split * yw + yg) * a.part_rows + xi - a.part_first;
        const bool direct = at.whole || a.part == nullptr;
        constexpr bool kBack = kScaled || kHalfBits;
        const float back = kBack && pscale[b] > 0.f ? 1.f / pscale[b] : kBack ? 0.f : 1.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = 32 * (db0 + d) + 8 * g + 4 * half;
                float4 v = make_float4(acc[b][d][4 * g], acc[b][d][4 * g + 1],
                                       acc[b][d][4 * g + 2], acc[b][d][4 * g + 3]);
                if constexpr (kBack) v = scale4(back, v);
                if (!direct) {
                    float4* p = reinterpret_cast<float4*>(a.part + row * a.dp + col);
                    *p = a.first ? v : add4(*p, v);
                } else if (a.out != nullptr && xi < a.x_rows && col < a.dim) {
                    store_out(static_cast<E*>(a.out) + xi * a.dim + col, v, a.scale, a.out_vec);
                }
            }
        if (!ROWS && blockIdx.y == 0 && a.want_bias) {
            const float v = bias[b] + __shfl_xor(bias[b], 32);
            if (half == 0) {
                if (!direct) a.bias_part[row] = v;
                else if (xi < a.x_rows) a.bias_out[xi] = v * a.scale;
            }
        }
    }
}

// Both gradients in one launch, the classes' workgroups first: one's last workgroups
// share the card with the other's first.
//
// Bound by the matrix cores and what stands between their products.  4096 x 1e6 x
// 128 bf16: 3540 to 3730 us by machine and data, 1.12 to 1.18 PFLOP/s over the four
// products (S twice); the matrix cores
// are busy 61% of the time, a SIMD issues vector instructions for another 47% of it
// (they overlap across three waves), and the clock stands at about 1.8 GHz under
// that load: the same calls on zeros take 22% less.  A library product of bf16
// matrices of 8192 reaches 1.4 to 1.6 PFLOP/s.  fp32, three products of halves for
// each: 3001 x 50021 x 256 1046 to 1196 us, 257 to 294 TFLOP/s (the library's fp32
// product: 154).  One wave per SIMD is all that X and the sums leave there, so that the
// exponentials run with the matrix cores idle: 42% busy.
//
// Measured against: workgroups of 4 waves with 128-column bf16 rows, dw and dh 2054 and
// 2140 us where 12 waves take 1881 and 2019 (fewer copies of the same Y records);
// dw at 1024 x 10000 x 32 with at least four tiles a wave and split 27 us, eight 24.
template <typename E, int ND, int XB, int WAVES, int OCC, bool STAGED, bool ANSWER>
__global__ __launch_bounds__(WAVES * 64) __attribute__((amdgpu_waves_per_eu(OCC, OCC)))
void k_sm_grad(PassArgs classes, PassArgs rows, int32_t class_blocks) {
    extern __shared__ __align__(16) uint8_t lds[];
    const int32_t b = blockIdx.x;
    if (b < class_blocks) grad_block<E, ND, XB, WAVES, STAGED, false, ANSWER>(classes, b, lds);
    else grad_block<E, ND, XB, WAVES, STAGED, true, ANSWER>(rows, b - class_blocks, lds);
}

// Partial results to be joined: `rows` rows from a slot each, part_rows apart.  Bound
// by memory and the launch: 17 us behind gradients of 3.8 ms, 4 us behind the smallest.
struct JoinArgs {
    const float* part;
    const float* bias_part;
    void* out;
    float* bias_out;
    int64_t part_rows, rows;
    int32_t slots, lanes;  // threads that share an output
    int64_t blocks;        // workgroups
    bool vec;
};

// The slots of four columns (or a bias), in an order that the sizes fix: LANES
// threads take every LANES-th, then add up.
template <typename E, int LANES>
__device__ __forceinline__ void join_slots(const JoinArgs& a, int64_t block, int dp, int dim,
                                           float scale) {
    const int64_t i = (block * kBlock + threadIdx.x) / LANES;
    const int lane = threadIdx.x % LANES;
    const int q = dim / 4;
    if (a.out != nullptr && i < a.rows * q) {
        const int64_t row = i / q;
        const int col = (int)(i % q) * 4;
        float4 v = zero4();
#pragma unroll 4
        for (int s = lane; s < a.slots; s += LANES)
            v = add4(v, *reinterpret_cast<const float4*>(a.part + (s * a.part_rows + row) * dp +
                                                         col));
        v = make_float4(group_sum<LANES>(v.x), group_sum<LANES>(v.y), group_sum<LANES>(v.z),
                        group_sum<LANES>(v.w));
        if (lane == 0) store_out(static_cast<E*>(a.out) + row * dim + col, v, scale, a.vec);
    }
    if (a.bias_out != nullptr && i < a.rows) {
        float v = 0.f;
#pragma unroll 4
        for (int s = lane; s < a.slots; s += LANES) v += a.bias_part[s * a.part_rows + i];
        v = group_sum<LANES>(v);
        if (lane == 0) a.bias_out[i] = v * scale;
    }
}

// One or two sets of partial results.
template <typename E>
__global__ __launch_bounds__(kBlock) void k_sm_join(JoinArgs a, JoinArgs b, int dp, int dim,
                                                    float scale, int64_t first) {
    int64_t block = first + blockIdx.x;
    const bool second = block >= a.blocks;
    const JoinArgs& k = second ? b : a;
    if (second) block -= a.blocks;
    if (k.lanes == 16) join_slots<E, 16>(k, block, dp, dim, scale);
    else join_slots<E, 1>(k, block, dp, dim, scale);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Rows that do not go through LDS: waves that wait for each other's loads less.
template <typename E, int ND, bool GRAD, bool STAGED, bool ANSWER = false>
constexpr int pass_occ() {
    return STAGED ? Shape<E, ND, GRAD, ANSWER>::kOcc : ND > 8 ? 1 : 2;
}
template <typename E, int ND, bool GRAD, bool STAGED, bool ANSWER = false>
constexpr int pass_waves() {
    return STAGED ? Shape<E, ND, GRAD, ANSWER>::kWaves
                  : 4 * pass_occ<E, ND, GRAD, STAGED, ANSWER>();
}

// Blocks of 32 columns that the kernels are made for.
inline int made_for(int nd) {
    for (int k : {1, 2, 3, 4, 6, 8, 10, 12, 16})
        if (nd <= k) return k;
    return 0;
}

constexpr int kSmLds = 152 * 1024;

struct Layout {
    int32_t x_groups, stage;
    int64_t x_blocks, x_whole, splits, per;
    int64_t slots, part_first, part_rows;  // partial results
};

constexpr int64_t kCus = 256;

// Workgroups along X and splits of Y.  With x_blocks above the card's places
// (`resident` workgroups of a CU), whole rounds of them take all of Y (where
// `whole` allows it) and what is left over is split; else all are.  A split has at
// least `least` tiles a wave; there are at most kSmPartRows partial rows (or one
// slot's).  Of the numbers of splits, the fewest that come within 3% of the
// shortest: r workgroups of 1 / s each take ceil(r s / places) / s, and a start that
// costs about as much as four tiles.  Each gradient is laid out as if it had the card
// to itself, though both share a launch and one's end overlaps the other's start.
Layout lay_out(int64_t x_tiles, int64_t y_tiles, int xb, int waves, int resident, int rec_bytes,
               bool staged, bool whole, int least) {
    Layout l{};
    const int64_t groups = div_up(x_tiles, xb);
    int64_t stage = staged ? kSmLds / 2 / resident / rec_bytes : waves;
    if (stage > 2 * waves) stage = 2 * waves;
    if (stage < 1) stage = 1;
    int g = waves;
    while (g > 1 && g / 2 >= groups && waves / (g / 2) <= stage) g /= 2;
    l.x_groups = g;
    const int yw = waves / g;
    l.x_blocks = div_up(groups, g);
    const int64_t places = kCus * resident;
    if (whole && yw == 1) l.x_whole = l.x_blocks / places * places;
    const int64_t left = l.x_blocks - l.x_whole;
    l.part_first = l.x_whole * g * xb * 32;
    l.part_rows = x_tiles * 32 - l.part_first;
    int64_t want = 1;
    if (left > 0) {
        int64_t most = y_tiles / (least * yw);
        const int64_t room = kSmPartRows / (l.part_rows * yw);
        if (most > room) most = room;
        double best = 1e30;
        for (int64_t s = 1; s <= most || s == 1; ++s) {
            const double time = (double)div_up(left * s, places) *
                                (1.0 / (double)s + 4.0 / (double)y_tiles);
            if (time < 0.97 * best) {
                best = time;
                want = s;
            }
        }
    }
    l.per = div_up(y_tiles, want);
    l.splits = div_up(y_tiles, l.per);
    l.slots = left > 0 ? l.splits * yw : 0;
    // as much of LDS as there is, in whole rounds of the waves along Y: a barrier
    // brings the waves into step, and their products then wait for each other
    l.stage = (int32_t)(stage / yw * yw);
    return l;
}

#define HUGE_SM_ND(ND_, ...)                            \
    switch (ND_) {                                      \
        case 1: { constexpr int ND = 1; __VA_ARGS__; } break; \
        case 2: { constexpr int ND = 2; __VA_ARGS__; } break; \
        case 3: { constexpr int ND = 3; __VA_ARGS__; } break; \
        case 4: { constexpr int ND = 4; __VA_ARGS__; } break; \
        case 6: { constexpr int ND = 6; __VA_ARGS__; } break; \
        case 8: { constexpr int ND = 8; __VA_ARGS__; } break; \
        case 10: { constexpr int ND = 10; __VA_ARGS__; } break; \
        case 12: { constexpr int ND = 12; __VA_ARGS__; } break; \
        case 16: { constexpr int ND = 16; __VA_ARGS__; } break; \
        default: return hipErrorInvalidValue;           \
    }

#define SM_TRY(expr)                        \
    do {                                    \
        const hipError_t e_ = (expr);       \
        if (e_ != hipSuccess) return e_;    \
    } while (0)

// Fills in the layout of a pass.
template <typename E, int ND, bool GRAD, bool STAGED, bool DIRECT, bool ANSWER = false>
Layout fit_pass(const SoftmaxPlan& p, bool rows, PassArgs& a) {
    using S = Shape<E, ND, GRAD, ANSWER>;
    const int rec = DIRECT ? 2 * ND * 1024 : record_bytes(p.dp / 16, p.parts, a.forms);
    const int occ = pass_occ<E, ND, GRAD, STAGED, ANSWER>();
    const int waves = pass_waves<E, ND, GRAD, STAGED, ANSWER>();
    // all pieces of the classes are laid out as the first, whose partial results they
    // add to
    const Layout l =
        lay_out(a.x_tiles, rows ? p.piece / kSmTile : a.y_tiles, STAGED ? S::kXB : 1, waves,
                occ * 4 / waves, rec, STAGED, GRAD && (!rows || p.piece >= p.classes),
                GRAD ? 8 : 4);
    a.x_groups = l.x_groups, a.stage = l.stage, a.x_blocks = (int32_t)l.x_blocks;
    a.x_whole = (int32_t)l.x_whole, a.splits = (int32_t)l.splits, a.per = l.per;
    a.part_first = l.part_first, a.part_rows = l.part_rows;
    a.nfrag = p.dp / 16, a.kd = p.kd, a.dp = p.dp, a.dim = p.dim;
    a.lds = !STAGED ? 0 : S::kHalves ? rec : 2 * l.stage * rec;
    a.grid = place_grid(l.x_blocks, l.x_whole, l.splits);
    return l;
}

template <typename E, int ND, bool STAGED, bool DIRECT, bool ANSWER>
hipError_t lse_pass(const SoftmaxPlan& p, PassArgs a, bool rows, int64_t* slots, hipStream_t s) {
    constexpr int kXB = STAGED ? Shape<E, ND, false, ANSWER>::kXB : 1;
    constexpr int kOcc = pass_occ<E, ND, false, STAGED, ANSWER>();
    constexpr int kWaves = pass_waves<E, ND, false, STAGED, ANSWER>();
    constexpr auto* kKernel = &k_sm_lse<E, ND, kXB, kWaves, kOcc, STAGED, DIRECT, ANSWER>;
    *slots = fit_pass<E, ND, false, STAGED, DIRECT, ANSWER>(p, rows, a).slots;
    if (a.lds > 64 * 1024) SM_TRY(allow_lds<kKernel>(kSmLds));
    kKernel<<<dim3((uint32_t)a.grid), kWaves * 64, a.lds, s>>>(a);
    return hipGetLastError();
}

// The pass of the loss.  rows: the classes come in pieces; else all at once.
template <typename E, bool ANSWER = false>
hipError_t lse_pass(const SoftmaxPlan& p, const PassArgs& a, bool rows, int64_t* slots,
                    hipStream_t s) {
    HUGE_SM_ND(p.nd, {
        if constexpr (sizeof(E) == 2)
            if (a.y_rows != nullptr) return lse_pass<E, ND, true, true, ANSWER>(p, a, rows, slots, s);
        if (p.chunks == 1) return lse_pass<E, ND, true, false, ANSWER>(p, a, rows, slots, s);
        if constexpr (ND == 8) return lse_pass<E, ND, false, false, ANSWER>(p, a, rows, slots, s);
    })
    return hipErrorInvalidValue;
}

template <typename E, int ND, bool STAGED, bool ANSWER, typename Fit>
hipError_t grad_pass(const SoftmaxPlan& p, PassArgs classes, PassArgs rows, Fit fit,
                     hipStream_t s) {
    constexpr int kXB = STAGED ? Shape<E, ND, true>::kXB : 1;
    constexpr int kOcc = pass_occ<E, ND, true, STAGED>();
    constexpr int kWaves = pass_waves<E, ND, true, STAGED>();
    constexpr auto* kKernel = &k_sm_grad<E, ND, kXB, kWaves, kOcc, STAGED, ANSWER>;
    Layout lc{}, lr{};
    if (classes.x != nullptr) lc = fit_pass<E, ND, true, STAGED, false>(p, false, classes);
    if (rows.x != nullptr) lr = fit_pass<E, ND, true, STAGED, false>(p, true, rows);
    fit(classes, lc, rows, lr);
    const int lds = classes.lds > rows.lds ? classes.lds : rows.lds;
    if (lds > 64 * 1024) SM_TRY(allow_lds<kKernel>(kSmLds));
    const dim3 grid((uint32_t)(classes.grid + rows.grid), (uint32_t)p.chunks);
    kKernel<<<grid, kWaves * 64, lds, s>>>(classes, rows, (int32_t)classes.grid);
    return hipGetLastError();
}

// The passes of the gradients; one whose x is null is left out.  fit sets the places
// of the partial results from the layouts.
template <typename E, bool ANSWER, typename Fit>
hipError_t grad_pass(const SoftmaxPlan& p, const PassArgs& classes, const PassArgs& rows, Fit fit,
                     hipStream_t s) {
    HUGE_SM_ND(p.nd, {
        if constexpr (Shape<E, ND, true>::kStaged) {
            if (p.chunks == 1) return grad_pass<E, ND, true, ANSWER>(p, classes, rows, fit, s);
            // wider rows: at least half of the largest ND in each of two chunks or more
            if constexpr (ND >= 6 && !Shape<E, ND, true>::kHalves)
                return grad_pass<E, ND, false, ANSWER>(p, classes, rows, fit, s);
        }
    })
    return hipErrorInvalidValue;
}

// Work that may be more than the 2^32 - 1 threads of a launch (2^28 rows of 16, 2^24 rows
// of 1024 columns) goes in launches of up to kLaunchBlocks workgroups of kBlock
// threads, each told its first.
constexpr int64_t kLaunchBlocks = (int64_t)1 << 23;

template <typename Launch>
hipError_t in_launches(int64_t blocks, Launch launch) {
    for (int64_t first = 0; first < blocks; first += kLaunchBlocks) {
        const int64_t left = blocks - first;
        launch(dim3((uint32_t)(left < kLaunchBlocks ? left : kLaunchBlocks)), first);
        SM_TRY(hipGetLastError());
    }
    return hipSuccess;
}

bool fours(const void* m, int64_t ld, size_t elem) {
    return (reinterpret_cast<uintptr_t>(m) & (4 * elem - 1)) == 0 && ld % 4 == 0;
}

// Packs a piece of the classes, and before the first the rows.
template <typename E, bool ANSWER = false, bool CODES = false>
hipError_t pack(const SoftmaxPlan& p, const SoftmaxArgs& a, int64_t c0, int64_t count, int forms,
                hipStream_t s, bool rows = true) {
    PackArgs w{}, h{};
    w.m = a.w, w.ld = a.ld_w, w.first = c0, w.count = count, w.tiles = div_up(count, kSmTile);
    w.out = a.ws + p.w, w.classes = true, w.vec = fours(a.w, a.ld_w, CODES ? 1 : sizeof(E));
    w.scales = a.w_scales, w.ld_scales = a.ld_scales;
    h.m = a.h, h.ld = a.ld_h, h.count = a.n;
    h.tiles = c0 == 0 && rows ? p.rows_pad / kSmTile : 0;
    h.out = a.ws + p.h, h.vec = fours(a.h, a.ld_h, sizeof(E));
    return in_launches(w.tiles + h.tiles, [&](dim3 grid, int64_t first) {
        k_sm_pack<E, ANSWER, CODES><<<grid, kBlock, 0, s>>>(a, w, h, p.dp / 16, forms, first);
    });
}

// The loss of few rows: up to 64 whose operands fit kFewLds.  Above that the tables'
// packing is paid for by the faster products.  Where n rows are few, fewer are too.
template <typename E, bool CODES = false>
int few_blocks(int64_t n, int32_t dim) {
    for (int nb = 1; nb <= 4; nb <<= 1)
        if (n <= 16 * nb) return few_operands<E, CODES>(dim) * nb * 1024 <= kFewLds<E> ? nb : 0;
    return 0;
}

// Workgroups of it: each leaves an entry per row.  Answers take as many as the card holds
// at once (by registers: four waves per SIMD, five of a table in 8 bits; by LDS), so that
// none starts behind another and what joins their entries has few: 38 x 300007 x 256 fp32 80 us
// with 512, 83 with 1024, 98 with 2048; 1 x 1e6 x 128 in 8 bits 32.4 with 1280, 33.7 with
// 2048, 38.8 with 1536.
template <typename E, int NB, bool ANSWER, bool CODES, bool THIRDS>
int64_t few_grid(int64_t classes, int32_t dim) {
    const int64_t need = div_up(div_up(classes, 16), few_waves(NB));
    int64_t most = 2048;
    if constexpr (ANSWER) {
        const int lds = (few_kb<E, CODES, THIRDS>(dim) + 2) * NB * 1024;  // with s_part
        int64_t at_once = NB == 1 ? (CODES ? 5 : 4) : 2;
        if (at_once > 160 * 1024 / lds) at_once = 160 * 1024 / lds;
        most = kCus * at_once;
    }
    return need < most ? need : most;
}

// of answers: the entries of a row are all_slots, these from slot0 on.
template <typename E, int NB, bool ANSWER = false, bool CODES = false, bool THIRDS = false>
hipError_t few_pass(const SoftmaxArgs& a, void* part, int64_t* slots, hipStream_t s,
                    float* best = nullptr, int64_t all_slots = 0, int64_t slot0 = 0) {
    constexpr int kWaves = few_waves(NB);
    const int64_t tiles = div_up(a.classes, 16);
    const int64_t blocks = few_grid<E, NB, ANSWER, CODES, THIRDS>(a.classes, a.dim);
    const int lds = few_kb<E, CODES, THIRDS>(a.dim) * NB * 1024;
    auto go = [&](auto bytes) {
        constexpr auto* kKernel = &k_sm_few<E, NB, decltype(bytes)::value, ANSWER, CODES, THIRDS>;
        if (lds > 60 * 1024) SM_TRY(allow_lds<kKernel>(kFewLds<E>));
        kKernel<<<dim3((uint32_t)blocks), kWaves * 64, lds, s>>>(a, tiles, part, 16 * NB, all_slots, slot0, best);
        return hipGetLastError();
    };
    *slots = blocks;
    if (a.vec16) return go(std::integral_constant<int, 16>{});
    if constexpr (CODES) {
        if (a.vec) return go(std::integral_constant<int, 4>{});
        return go(std::integral_constant<int, 1>{});
    } else {
        if constexpr (sizeof(E) == 2)
            if (a.vec) return go(std::integral_constant<int, 8>{});
        return go(std::integral_constant<int, sizeof(E)>{});
    }
}

// The partial results of the rows from lay.part_first on, of `rows`.
template <typename E>
JoinArgs to_join(const SoftmaxPlan& p, const float* part, const Layout& lay, int64_t rows,
                 void* out, const float* bias_part, float* bias_out) {
    JoinArgs j{};
    j.rows = rows - lay.part_first;
    if (j.rows <= 0) return JoinArgs{};
    j.part = part, j.bias_part = bias_part, j.part_rows = lay.part_rows;
    j.out = out == nullptr ? nullptr : static_cast<E*>(out) + lay.part_first * p.dim;
    j.bias_out = bias_out == nullptr ? nullptr : bias_out + lay.part_first;
    j.vec = fours(j.out, 0, sizeof(E));
    j.slots = (int32_t)lay.slots;
    const int64_t work = out != nullptr ? j.rows * (p.dim / 4) : j.rows;
    // few outputs of many slots: 16 threads each.  Both joins of 100003 x 100 x 32 bf16
    // take 8 us, 52 with one thread each; of 16384 x 1000 x 128 11 us, 16 with one each
    // and 29 with 16 each; of 8192 x 8192 x 64, where it errs, 15 with 12 and 15
    j.lanes = work < (1 << 18) && lay.slots >= 16 ? 16 : 1;
    j.blocks = div_up(work * j.lanes, kBlock);
    return j;
}

template <typename E>
hipError_t join(const SoftmaxPlan& p, const JoinArgs& a, const JoinArgs& b, float scale,
                hipStream_t s) {
    return in_launches(a.blocks + b.blocks, [&](dim3 grid, int64_t first) {
        k_sm_join<E><<<grid, kBlock, 0, s>>>(a, b, p.dp, p.dim, scale, first);
    });
}

template <typename E, bool ANSWER = false>
hipError_t softmax_grad(const SoftmaxArgs& a, hipStream_t s) {
    const SoftmaxPlan p = softmax_plan(a.classes, a.n, a.dim, a.dtype, true);
    const int64_t x_tiles = p.rows_pad / kSmTile;
    float* class_part = reinterpret_cast<float*>(a.ws + p.part);
    float* row_part = reinterpret_cast<float*>(a.ws + p.row_part);
    JoinArgs row_join{};
    for (int64_t c0 = 0; c0 < a.classes; c0 += p.piece) {
        const int64_t count = a.classes - c0 < p.piece ? a.classes - c0 : p.piece;
        const int64_t w_tiles = div_up(count, kSmTile);
        SM_TRY((pack<E, ANSWER>(p, a, c0, count, 2, s)));
        PassArgs c{}, r{};
        c.class0 = r.class0 = c0, c.scale = r.scale = a.scale, c.forms = r.forms = 2;
        if (a.dw != nullptr || a.dbias != nullptr) {
            // the second product is formed also where only the bias is wanted
            c.x = a.ws + p.w, c.y = a.ws + p.h, c.x_tiles = w_tiles, c.y_tiles = x_tiles;
            c.x_rows = count, c.first = true, c.want_bias = a.dbias != nullptr;
            c.out = a.dw == nullptr ? nullptr : static_cast<E*>(a.dw) + c0 * p.dim;
            c.bias_out = a.dbias == nullptr ? nullptr : a.dbias + c0;
            c.out_vec = fours(c.out, 0, sizeof(E));
        }
        if (a.dh != nullptr) {
            r.x = a.ws + p.h, r.y = a.ws + p.w, r.x_tiles = x_tiles, r.y_tiles = w_tiles;
            r.x_rows = a.n, r.first = c0 == 0, r.out = a.dh, r.out_vec = fours(a.dh, 0, sizeof(E));
        }
        JoinArgs class_join{};
        SM_TRY((grad_pass<E, ANSWER>(
            p, c, r,
            [&](PassArgs& q, const Layout& lc, PassArgs& t, const Layout& lr) {
                if (lc.slots > 1) {
                    q.part = class_part;
                    q.bias_part = class_part + lc.slots * lc.part_rows * p.dp;
                    class_join = to_join<E>(p, q.part, lc, count, q.out, q.bias_part, q.bias_out);
                }
                // the rows' sums stay from piece to piece
                if (lr.slots > 1 || (t.x != nullptr && p.piece < a.classes)) {
                    t.part = row_part;
                    row_join = to_join<E>(p, row_part, lr, a.n, a.dh, nullptr, nullptr);
                }
            },
            s)));
        const bool last = c0 + p.piece >= a.classes;
        SM_TRY(join<E>(p, class_join, last ? row_join : JoinArgs{}, a.scale, s));
    }
    return hipSuccess;
}

}  // namespace

}  // namespace huge
