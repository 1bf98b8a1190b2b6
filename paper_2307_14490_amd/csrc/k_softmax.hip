// The exact softmax loss over a large vocabulary and its gradient, without the
// logits in memory.
//
// With S = H W' + bias, the loss needs lse_i = log sum_j exp S_ij, and the gradient
// G = c (exp(S - lse) - onehot) only in the products G W and G' H.  Each of the
// three passes forms a 32 x 32 tile of S on the matrix cores, uses it in
// registers and drops it: the loss keeps a running maximum and sum per row, the
// two gradients multiply the tile at once.  S is formed three times in all, which
// at the widths of embeddings costs less than a round trip of its elements
// through memory: at 4 + 4 bytes an element that would be about 0.6 clocks of a
// CU, and 2 D flops are 0.06 at D = 128.
//
// Both gradients are one kernel: X are the rows whose gradient is formed (one
// tile or two per wave, in registers), Y the rows that are summed over.  A tile
// is computed with Y as the rows and X as the columns of the product, so that a
// lane holds 16 elements of one X row: sums, maxima and scales per X row need no
// exchange between lanes, and the tile in its place is the second operand of the
// product with Y' (whose operand holds Y's rows in the order in which the first
// product leaves them).  The terms per Y row (a class's bias; a row's
// log weight - lse) are the initial value of the tile.
//
// Operands are packed before: R form (rows as they enter S) and T form (rows as
// they enter the second product), tiles of 32 rows, each 1 KB block being one
// operand of a 32x32x16 product in lane order.  fp32 rows are three bf16 parts,
// whose sum is the fp32 value exactly, and the six products of parts that are
// not below 2^-24 of the whole are formed; so are those of the tile in the
// second product.  bf16 rows are one part, and the tile is rounded to bf16
// (after the label is subtracted, so that a probability near one keeps its small
// complement): an error of 2^-8 of each term at most, as in the rounding of the result.
#include <math.h>

#include "device.hpp"
#include "head.hpp"

namespace huge {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Row of a product's register i in lane half h (the column is lane % 32).
__device__ __forceinline__ int tile_row(int i, int h) { return 8 * (i / 4) + 4 * h + i % 4; }

template <int PARTS>
struct Parts {
    bf16x8 p[PARTS];
};

// The parts of eight values: each the nearest bf16 to what the ones before leave.
template <int PARTS>
__device__ __forceinline__ Parts<PARTS> split(f32x8 v) {
    Parts<PARTS> r;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
        r.p[k] = __builtin_convertvector(v, bf16x8);
        if (k + 1 < PARTS) v -= __builtin_convertvector(r.p[k], f32x8);
    }
    return r;
}

// c + a b, over the products of parts that reach 2^-24 of the whole.
template <int PARTS>
__device__ __forceinline__ f32x16 mfma_parts(const Parts<PARTS>& a, const Parts<PARTS>& b,
                                             f32x16 c) {
    if constexpr (PARTS == 3) {
        c = mfma(a.p[2], b.p[0], c);
        c = mfma(a.p[0], b.p[2], c);
        c = mfma(a.p[1], b.p[1], c);
        c = mfma(a.p[1], b.p[0], c);
        c = mfma(a.p[0], b.p[1], c);
    }
    return mfma(a.p[0], b.p[0], c);
}

// Operand `f` of a packed tile: parts lie `stride` operands apart.
template <int PARTS>
__device__ __forceinline__ Parts<PARTS> load_frag(const bf16x8* __restrict__ tile, int f,
                                                  int stride, int lane) {
    Parts<PARTS> r;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) r.p[k] = tile[(k * stride + f) * 64 + lane];
    return r;
}

__device__ __forceinline__ void set_status(int32_t* status, int32_t code) {
    atomicCAS(status, 0, code);
}

// ---------------------------------------------------------------------------
// Packing
// ---------------------------------------------------------------------------
struct PackArgs {
    const void* m;
    int64_t ld, first, rows;  // rows first .. first + rows of the matrix
    int dim, nfrag;           // operands of a tile and part, one form
    const float* bias;        // classes: the tile's terms are these (or 0), -inf past the end
    float* term;              // or null
    const float* live;        // rows: those at -inf are packed as zeros
    bf16x8* r;
    bf16x8* t;                // or null
};

// A workgroup packs 32 rows x 128 columns.
template <typename E, int PARTS>
__global__ __launch_bounds__(kBlock) void k_sm_pack(PackArgs a) {
    __shared__ float s[32][132];
    __shared__ bool s_out[32];
    const int64_t tile = blockIdx.x;
    const int col0 = blockIdx.y * 128;
    if (threadIdx.x < 32) {
        const int64_t r = tile * 32 + threadIdx.x;
        bool out = r >= a.rows;
        if (a.term != nullptr) {
            const float b = out ? -INFINITY : a.bias == nullptr ? 0.f : a.bias[a.first + r];
            out = b == -INFINITY;
            if (blockIdx.y == 0) a.term[r] = b;
        }
        if (a.live != nullptr && !out) out = a.live[r] == -INFINITY;
        s_out[threadIdx.x] = out;
    }
    __syncthreads();
    const E* m = static_cast<const E*>(a.m);
    for (int j = threadIdx.x; j < 32 * 128; j += kBlock) {
        const int row = j >> 7, col = j & 127;
        float v = 0.f;
        if (!s_out[row] && col0 + col < a.dim) {
            const E e = m[(a.first + tile * 32 + row) * a.ld + col0 + col];
            if constexpr (sizeof(E) == 4) v = e;
            else v = __uint_as_float((uint32_t)e << 16);
        }
        s[row][col] = v;
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int nd = a.nfrag / 2;
    for (int k = wave; k < 8; k += 4) {
        const int f = blockIdx.y * 8 + k;
        if (f < a.nfrag) {
            f32x8 v;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = s[lane & 31][16 * k + 8 * half + j];
            const Parts<PARTS> p = split<PARTS>(v);
#pragma unroll
            for (int q = 0; q < PARTS; ++q)
                a.r[((tile * PARTS + q) * a.nfrag + f) * 64 + lane] = p.p[q];
        }
        const int db = blockIdx.y * 4 + (k & 3), t = k >> 2;
        if (a.t != nullptr && db < nd) {
            f32x8 v;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = s[16 * t + tile_row(j, half)][32 * (k & 3) + (lane & 31)];
            const Parts<PARTS> p = split<PARTS>(v);
#pragma unroll
            for (int q = 0; q < PARTS; ++q)
                a.t[((tile * PARTS + q) * a.nfrag + t * nd + db) * 64 + lane] = p.p[q];
        }
    }
}

// ---------------------------------------------------------------------------
// Loss: running maximum and sum
// ---------------------------------------------------------------------------
struct LseArgs {
    const bf16x8* x;     // rows, R form
    const bf16x8* y;     // classes, R form
    const float* term;   // a class's bias, -inf for those that are out
    int64_t x_tiles, y_tiles, per;  // y tiles of a split
    int nfrag, kd;
    bool first;          // the first piece of the classes
    float2* part;        // [split][32 x_tiles]: maximum and sum
};

// exp(a - b) for a <= b, 0 where a is -inf (also if b is).
__device__ __forceinline__ float exp_below(float a, float b) {
    return a == -INFINITY ? 0.f : exp2f((a - b) * kLog2e);
}

template <int ND, int PARTS, bool XREG>
__global__ __launch_bounds__(kSmWaves * 64) void k_sm_lse(LseArgs a) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int64_t xt = (int64_t)blockIdx.x * kSmWaves + (threadIdx.x >> 6);
    if (xt >= a.x_tiles) return;
    const bf16x8* xp = a.x + xt * PARTS * a.nfrag * 64;
    constexpr int KD = 2 * ND;
    Parts<PARTS> x[XREG ? KD : 1];
    if constexpr (XREG) {
#pragma unroll
        for (int k = 0; k < KD; ++k) x[k] = load_frag<PARTS>(xp, k, a.nfrag, lane);
    }
    const int64_t y0 = (int64_t)blockIdx.y * a.per;
    const int64_t y1 = y0 + a.per < a.y_tiles ? y0 + a.per : a.y_tiles;
    float2* out = a.part + (int64_t)blockIdx.y * a.x_tiles * 32 + xt * 32 + (lane & 31);
    float top = -INFINITY, sum = 0.f;
    for (int64_t yt = y0; yt < y1; ++yt) {
        const bf16x8* yp = a.y + yt * PARTS * a.nfrag * 64;
        const float4* term = reinterpret_cast<const float4*>(a.term + yt * 32) + half;
        f32x16 c;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 b = term[2 * g];
            c[4 * g] = b.x, c[4 * g + 1] = b.y, c[4 * g + 2] = b.z, c[4 * g + 3] = b.w;
        }
        if constexpr (XREG) {
#pragma unroll
            for (int k = 0; k < KD; ++k)
                c = mfma_parts<PARTS>(load_frag<PARTS>(yp, k, a.nfrag, lane), x[k], c);
        } else {
            for (int k = 0; k < a.kd; ++k)
                c = mfma_parts<PARTS>(load_frag<PARTS>(yp, k, a.nfrag, lane),
                                      load_frag<PARTS>(xp, k, a.nfrag, lane), c);
        }
        float m = top;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = fmaxf(m, c[i]);
        const float ref = m == -INFINITY ? 0.f : m;
        sum *= exp_below(top, ref);
        top = m;
        const float sub = -ref * kLog2e;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(fmaf(c[i], kLog2e, sub));
    }
    // the halves hold different classes of the same row
    const float top2 = __shfl_xor(top, 32), sum2 = __shfl_xor(sum, 32);
    float m = fmaxf(top, top2);
    sum = sum * exp_below(top, m) + sum2 * exp_below(top2, m);
    if (half == 0) {
        if (!a.first) {
            const float2 p = *out;
            const float mm = fmaxf(m, p.x);
            sum = sum * exp_below(m, mm) + p.y * exp_below(p.x, mm);
            m = mm;
        }
        *out = make_float2(m, sum);
    }
}

// lse and loss of a row, a wave each: the splits are joined in order, and the
// label's logit is formed from the rows themselves.
template <typename E>
__global__ __launch_bounds__(kBlock) void k_sm_loss(SoftmaxArgs a, const float2* __restrict__ part,
                                                    int splits, int64_t pad) {
    const int lane = threadIdx.x & 63;
    const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= a.n) return;
    float m = -INFINITY, sum = 0.f;
    bool nan = false;
    for (int s = lane; s < splits; s += 64) {
        const float2 p = part[(int64_t)s * pad + i];
        const float mm = fmaxf(m, p.x);
        nan |= p.y != p.y;
        sum = sum * exp_below(m, mm) + p.y * exp_below(p.x, mm);
        m = mm;
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const float m2 = __shfl_xor(m, off), s2 = __shfl_xor(sum, off);
        const float mm = fmaxf(m, m2);
        sum = sum * exp_below(m, mm) + s2 * exp_below(m2, mm);
        m = mm;
    }
    nan = __ballot(nan) != 0;
    const float lse = nan ? NAN : m == -INFINITY ? -INFINITY : m + logf(sum);
    const int32_t y = a.labels[i];
    const float c = a.weight == nullptr ? 1.f : a.weight[i];
    float loss = 0.f;
    if (y < -1 || y >= a.classes) {
        loss = NAN;
        if (lane == 0) set_status(a.status, -2);
    } else if (!(c >= 0.f && c < INFINITY)) {
        loss = NAN;
        if (lane == 0) set_status(a.status, -3);
    } else if (y >= 0 && c > 0.f) {
        const float b = a.bias == nullptr ? 0.f : a.bias[y];
        if (b != -INFINITY) {
            const E* h = static_cast<const E*>(a.h) + i * a.ld_h;
            const E* w = static_cast<const E*>(a.w) + (int64_t)y * a.ld_w;
            float dot = 0.f;
            for (int d = lane; d < a.dim; d += 64) {
                if constexpr (sizeof(E) == 4) dot = fmaf(h[d], w[d], dot);
                else dot = fmaf(__uint_as_float((uint32_t)h[d] << 16),
                                __uint_as_float((uint32_t)w[d] << 16), dot);
            }
            const float below = lse - (group_sum<64>(dot) + b);
            loss = c * (below < 0.f ? 0.f : below);  // rounding alone takes it below 0
        }
    }
    if (lane == 0) {
        a.lse[i] = lse;
        a.loss[i] = loss;
    }
}

__global__ __launch_bounds__(1024) void k_sm_sum(const float* __restrict__ loss, int64_t n,
                                                 double* __restrict__ out) {
    __shared__ double s[1024];
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) v += (double)loss[i];
    s[threadIdx.x] = v;
    __syncthreads();
    for (int k = 512; k > 0; k >>= 1) {
        if (threadIdx.x < k) s[threadIdx.x] += s[threadIdx.x + k];
        __syncthreads();
    }
    if (threadIdx.x == 0) *out = s[0];
}

// ---------------------------------------------------------------------------
// Gradients
// ---------------------------------------------------------------------------
// Per row: log weight - lse (-inf without a loss), the label (-1 then) and the
// weight, in whole tiles.
__global__ __launch_bounds__(kBlock) void k_sm_rows(SoftmaxArgs a, int64_t pad,
                                                    float* __restrict__ term,
                                                    int32_t* __restrict__ label,
                                                    float* __restrict__ cw) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= pad) return;
    float t = -INFINITY, c = 0.f;
    int32_t y = -1;
    if (i < a.n) {
        y = a.labels[i];
        c = a.weight == nullptr ? 1.f : a.weight[i];
        const bool bad_y = y < -1 || y >= a.classes, bad_c = !(c >= 0.f && c < INFINITY);
        if (bad_y) set_status(a.status, -2);
        else if (bad_c) set_status(a.status, -3);
        if (bad_y || bad_c || y < 0 || c == 0.f || (a.bias != nullptr && a.bias[y] == -INFINITY)) {
            y = -1;
            c = 0.f;
        } else {
            t = logf(c) - a.lse[i];
        }
    }
    term[i] = t;
    label[i] = y;
    cw[i] = c;
}

struct GradArgs {
    const bf16x8* xr;      // X, R form
    const bf16x8* yr;      // Y, R form and T form
    const bf16x8* yt;
    const float* xterm;    // what is added to the tile per X row and per Y row
    const float* yterm;
    const int32_t* label;  // of the rows (X or Y)
    const float* cw;
    int64_t class0;        // first class of the piece
    int64_t x_rows, x_tiles, y_tiles, per;
    int nfrag, kd, dp, dim;
    bool first;            // partial sums: written, else added to
    float* part;           // [split][32 x_tiles][dp], or null: to `out`
    float* bias_part;      // [split][32 x_tiles] (X: classes), or null
    void* out;             // x_rows x dim
    float* bias_out;
    float scale;
};

template <typename E>
__device__ __forceinline__ void store_out(E* p, float4 v, float scale) {
    // alignment of the element type is all that the caller owes
    const float q[4] = {v.x * scale, v.y * scale, v.z * scale, v.w * scale};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(E) == 4) p[e] = q[e];
        else p[e] = (bf16_t)float_to_bf16_bits(q[e]);
    }
}

// ROWS: X are the rows and Y the classes (dh), else X are the classes (dw).
template <typename E, int ND, int PARTS, bool ROWS, bool XREG>
__global__ __launch_bounds__(kSmWaves * 64) void k_sm_grad(GradArgs a) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int64_t xt = (int64_t)blockIdx.x * kSmWaves + (threadIdx.x >> 6);
    if (xt >= a.x_tiles) return;
    const int db0 = blockIdx.z * ND, nd = a.nfrag / 2;
    const bf16x8* xp = a.xr + xt * PARTS * a.nfrag * 64;
    constexpr int KD = 2 * ND;
    Parts<PARTS> x[XREG ? KD : 1];
    if constexpr (XREG) {
#pragma unroll
        for (int k = 0; k < KD; ++k) x[k] = load_frag<PARTS>(xp, k, a.nfrag, lane);
    }
    const int64_t xi = xt * 32 + (lane & 31);
    const float xterm = a.xterm[xi];
    // the label that this lane's elements are compared with: a class of this piece,
    // or (X: classes) the lane's class against each row's label
    const int64_t xl = ROWS ? (int64_t)a.label[xi] - a.class0 : a.class0 + xi;
    const float xc = ROWS ? a.cw[xi] : 0.f;
    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) acc[d] = f32x16{};
    float bias = 0.f;
    const int64_t y0 = (int64_t)blockIdx.y * a.per;
    const int64_t y1 = y0 + a.per < a.y_tiles ? y0 + a.per : a.y_tiles;
    for (int64_t yt = y0; yt < y1; ++yt) {
        const bf16x8* yp = a.yr + yt * PARTS * a.nfrag * 64;
        const bf16x8* tp = a.yt + yt * PARTS * a.nfrag * 64;
        const float4* term = reinterpret_cast<const float4*>(a.yterm + yt * 32) + half;
        f32x16 c;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 b = term[2 * g];
            c[4 * g] = b.x, c[4 * g + 1] = b.y, c[4 * g + 2] = b.z, c[4 * g + 3] = b.w;
        }
        if constexpr (XREG) {
#pragma unroll
            for (int k = 0; k < KD; ++k)
                c = mfma_parts<PARTS>(load_frag<PARTS>(yp, k, a.nfrag, lane), x[k], c);
        } else {
            for (int k = 0; k < a.kd; ++k)
                c = mfma_parts<PARTS>(load_frag<PARTS>(yp, k, a.nfrag, lane),
                                      load_frag<PARTS>(xp, k, a.nfrag, lane), c);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) c[i] = __builtin_amdgcn_exp2f((c[i] + xterm) * kLog2e);
        // the label's element, in the few tiles that hold one
        if constexpr (ROWS) {
            const int64_t at = xl - yt * 32;
            if (__ballot(at >= 0 && at < 32 && a.label[xi] >= 0) != 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (at == tile_row(i, half)) c[i] -= xc;
            }
        } else {
            const int32_t* lab = a.label + yt * 32;
            const int64_t at = (int64_t)lab[lane & 31] - (a.class0 + xt * 32);
            if (__ballot(at >= 0 && at < 32) != 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (lab[tile_row(i, half)] == xl) c[i] -= a.cw[yt * 32 + tile_row(i, half)];
            }
            if (a.bias_part != nullptr || a.bias_out != nullptr) {
#pragma unroll
                for (int i = 0; i < 16; ++i) bias += c[i];
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x8 v;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = c[8 * t + j];
            const Parts<PARTS> p = split<PARTS>(v);
#pragma unroll
            for (int d = 0; d < ND; ++d)
                acc[d] = mfma_parts<PARTS>(
                    load_frag<PARTS>(tp, t * nd + db0 + d, a.nfrag, lane), p, acc[d]);
        }
    }
    const int64_t row = (int64_t)blockIdx.y * a.x_tiles * 32 + xi;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = 32 * (db0 + d) + 8 * g + 4 * half;
            float4 v = make_float4(acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2],
                                   acc[d][4 * g + 3]);
            if (a.part != nullptr) {
                float4* p = reinterpret_cast<float4*>(a.part + row * a.dp + col);
                *p = a.first ? v : add4(*p, v);
            } else if (a.out != nullptr && xi < a.x_rows && col < a.dim) {
                store_out(static_cast<E*>(a.out) + xi * a.dim + col, v, a.scale);
            }
        }
    }
    if (!ROWS && blockIdx.z == 0) {
        bias += __shfl_xor(bias, 32);
        if (half == 0) {
            if (a.bias_part != nullptr) a.bias_part[row] = bias;
            else if (a.bias_out != nullptr && xi < a.x_rows) a.bias_out[xi] = bias * a.scale;
        }
    }
}

// The splits' partial sums, in order.
template <typename E>
__global__ __launch_bounds__(kBlock) void k_sm_join(const float* __restrict__ part, int splits,
                                                    int64_t rows_pad, int dp, int64_t rows,
                                                    int dim, float scale, E* __restrict__ out,
                                                    const float* __restrict__ bias_part,
                                                    float* __restrict__ bias_out) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    const int q = dim / 4;
    if (out != nullptr && i < rows * q) {
        const int64_t row = i / q;
        const int col = (int)(i % q) * 4;
        float4 v = zero4();
        for (int s = 0; s < splits; ++s)
            v = add4(v, *reinterpret_cast<const float4*>(part + (s * rows_pad + row) * dp + col));
        store_out(out + row * dim + col, v, scale);
    }
    if (bias_out != nullptr && i < rows) {
        float v = 0.f;
        for (int s = 0; s < splits; ++s) v += bias_part[s * rows_pad + i];
        bias_out[i] = v * scale;
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Splits {
    int64_t count, per;
};

// Enough workgroups to fill the card, from splits of the summed rows; not more
// rows of partial sums than kSmPartRows (or one split's).
Splits split_tiles(int64_t x_tiles, int64_t y_tiles) {
    const int64_t blocks = div_up(x_tiles, kSmWaves);
    int64_t want = div_up(1024, blocks);
    const int64_t room = kSmPartRows / (x_tiles * 32);
    if (want > room) want = room;
    if (want > y_tiles) want = y_tiles;
    if (want < 1) want = 1;
    const int64_t per = div_up(y_tiles, want);
    return {div_up(y_tiles, per), per};
}

#define HUGE_SM_ND(ND_, ...)                            \
    switch (ND_) {                                      \
        case 1: { constexpr int ND = 1; __VA_ARGS__; } break; \
        case 2: { constexpr int ND = 2; __VA_ARGS__; } break; \
        case 3: { constexpr int ND = 3; __VA_ARGS__; } break; \
        case 4: { constexpr int ND = 4; __VA_ARGS__; } break; \
        case 6: { constexpr int ND = 6; __VA_ARGS__; } break; \
        case 8: { constexpr int ND = 8; __VA_ARGS__; } break; \
        default: return hipErrorInvalidValue;           \
    }

template <typename E>
constexpr int kPartsOf = sizeof(E) == 4 ? 3 : 1;

template <typename E>
hipError_t pack(const SoftmaxPlan& p, PackArgs a, int64_t tiles, hipStream_t s) {
    a.dim = p.dim;
    a.nfrag = p.dp / 16;
    const dim3 grid((uint32_t)tiles, (uint32_t)div_up(p.dp, 128));
    k_sm_pack<E, kPartsOf<E>><<<grid, kBlock, 0, s>>>(a);
    return hipGetLastError();
}

template <typename E>
hipError_t lse_pass(const SoftmaxPlan& p, const LseArgs& a, int64_t splits, hipStream_t s) {
    const dim3 grid((uint32_t)div_up(a.x_tiles, kSmWaves), (uint32_t)splits);
    HUGE_SM_ND(p.nd, if (p.chunks == 1) {
        k_sm_lse<ND, kPartsOf<E>, true><<<grid, kSmWaves * 64, 0, s>>>(a);
    } else {
        k_sm_lse<ND, kPartsOf<E>, false><<<grid, kSmWaves * 64, 0, s>>>(a);
    })
    return hipGetLastError();
}

template <typename E, bool ROWS>
hipError_t grad_pass(const SoftmaxPlan& p, const GradArgs& a, int64_t splits, hipStream_t s) {
    const dim3 grid((uint32_t)div_up(a.x_tiles, kSmWaves), (uint32_t)splits, (uint32_t)p.chunks);
    HUGE_SM_ND(p.nd, if (p.chunks == 1) {
        k_sm_grad<E, ND, kPartsOf<E>, ROWS, true><<<grid, kSmWaves * 64, 0, s>>>(a);
    } else {
        k_sm_grad<E, ND, kPartsOf<E>, ROWS, false><<<grid, kSmWaves * 64, 0, s>>>(a);
    })
    return hipGetLastError();
}

#define SM_TRY(expr)                        \
    do {                                    \
        const hipError_t e_ = (expr);       \
        if (e_ != hipSuccess) return e_;    \
    } while (0)

template <typename E>
hipError_t softmax_loss(const SoftmaxArgs& a, hipStream_t s) {
    const SoftmaxPlan p = softmax_plan(a.classes, a.n, a.dim, a.dtype, false);
    auto at = [&](size_t off) { return a.ws + off; };
    const int64_t x_tiles = p.rows_pad / kSmTile;
    float2* part = reinterpret_cast<float2*>(at(p.part));
    PackArgs h{};
    h.m = a.h, h.ld = a.ld_h, h.rows = a.n;
    h.r = reinterpret_cast<bf16x8*>(at(p.hr));
    SM_TRY(pack<E>(p, h, x_tiles, s));
    const Splits sp = split_tiles(x_tiles, p.piece / kSmTile);
    for (int64_t c0 = 0; c0 < a.classes; c0 += p.piece) {
        const int64_t count = a.classes - c0 < p.piece ? a.classes - c0 : p.piece;
        PackArgs w{};
        w.m = a.w, w.ld = a.ld_w, w.first = c0, w.rows = count, w.bias = a.bias;
        w.term = reinterpret_cast<float*>(at(p.yterm));
        w.r = reinterpret_cast<bf16x8*>(at(p.wr));
        SM_TRY(pack<E>(p, w, div_up(count, kSmTile), s));
        LseArgs l{};
        l.x = h.r, l.y = w.r, l.term = w.term;
        l.x_tiles = x_tiles, l.y_tiles = div_up(count, kSmTile), l.per = sp.per;
        l.nfrag = p.dp / 16, l.kd = p.kd, l.first = c0 == 0, l.part = part;
        SM_TRY(lse_pass<E>(p, l, sp.count, s));
    }
    k_sm_loss<E><<<dim3((uint32_t)div_up(a.n, 4)), kBlock, 0, s>>>(a, part, (int)sp.count,
                                                                  p.rows_pad);
    SM_TRY(hipGetLastError());
    if (a.loss_sum != nullptr) {
        k_sm_sum<<<1, 1024, 0, s>>>(a.loss, a.n, a.loss_sum);
        SM_TRY(hipGetLastError());
    }
    return hipSuccess;
}

template <typename E>
hipError_t join(const SoftmaxPlan& p, const float* part, int64_t splits, int64_t rows_pad,
                int64_t rows, float scale, void* out, const float* bias_part, float* bias_out,
                hipStream_t s) {
    const int64_t work = out != nullptr ? rows * (p.dim / 4) : rows;
    k_sm_join<E><<<dim3((uint32_t)div_up(work, kBlock)), kBlock, 0, s>>>(
        part, (int)splits, rows_pad, p.dp, rows, p.dim, scale, static_cast<E*>(out), bias_part,
        bias_out);
    return hipGetLastError();
}

template <typename E>
hipError_t softmax_grad(const SoftmaxArgs& a, hipStream_t s) {
    const SoftmaxPlan p = softmax_plan(a.classes, a.n, a.dim, a.dtype, true);
    auto at = [&](size_t off) { return a.ws + off; };
    const int64_t x_tiles = p.rows_pad / kSmTile;
    float* row_term = reinterpret_cast<float*>(at(p.xrow));
    int32_t* label = reinterpret_cast<int32_t*>(at(p.xlab));
    float* cw = reinterpret_cast<float*>(at(p.xcw));
    float* part = reinterpret_cast<float*>(at(p.part));
    k_sm_rows<<<dim3((uint32_t)div_up(p.rows_pad, kBlock)), kBlock, 0, s>>>(a, p.rows_pad, row_term,
                                                                           label, cw);
    SM_TRY(hipGetLastError());
    PackArgs h{};
    h.m = a.h, h.ld = a.ld_h, h.rows = a.n, h.live = row_term;
    h.r = reinterpret_cast<bf16x8*>(at(p.hr));
    h.t = reinterpret_cast<bf16x8*>(at(p.ht));
    SM_TRY(pack<E>(p, h, x_tiles, s));
    const Splits sp = split_tiles(x_tiles, p.piece / kSmTile);
    const bool direct = sp.count == 1 && p.piece >= a.classes;
    for (int64_t c0 = 0; c0 < a.classes; c0 += p.piece) {
        const int64_t count = a.classes - c0 < p.piece ? a.classes - c0 : p.piece;
        const int64_t w_tiles = div_up(count, kSmTile);
        PackArgs w{};
        w.m = a.w, w.ld = a.ld_w, w.first = c0, w.rows = count, w.bias = a.bias;
        w.term = reinterpret_cast<float*>(at(p.yterm));
        w.r = reinterpret_cast<bf16x8*>(at(p.wr));
        w.t = reinterpret_cast<bf16x8*>(at(p.wt));
        SM_TRY(pack<E>(p, w, w_tiles, s));
        GradArgs g{};
        g.label = label, g.cw = cw, g.class0 = c0, g.scale = a.scale;
        g.nfrag = p.dp / 16, g.kd = p.kd, g.dp = p.dp, g.dim = p.dim;
        if (a.dw != nullptr || a.dbias != nullptr) {
            const Splits sw = split_tiles(w_tiles, x_tiles);
            g.xr = w.r, g.yr = h.r, g.yt = h.t, g.xterm = w.term, g.yterm = row_term;
            g.x_rows = count, g.x_tiles = w_tiles, g.y_tiles = x_tiles, g.per = sw.per;
            g.first = true;
            E* out = a.dw == nullptr ? nullptr : static_cast<E*>(a.dw) + c0 * p.dim;
            float* bias_out = a.dbias == nullptr ? nullptr : a.dbias + c0;
            // the second product is formed also where only the bias is wanted
            g.part = sw.count > 1 ? part : nullptr;
            g.bias_part = sw.count > 1 ? part + sw.count * w_tiles * 32 * p.dp : nullptr;
            g.out = out, g.bias_out = bias_out;
            SM_TRY((grad_pass<E, false>(p, g, sw.count, s)));
            if (sw.count > 1)
                SM_TRY(join<E>(p, part, sw.count, w_tiles * 32, count, a.scale, out, g.bias_part,
                               bias_out, s));
        }
        if (a.dh != nullptr) {
            // the partial sums of the rows lie behind those of the classes: they
            // stay from piece to piece
            g.xr = h.r, g.yr = w.r, g.yt = w.t, g.xterm = row_term, g.yterm = w.term;
            g.x_rows = a.n, g.x_tiles = x_tiles, g.y_tiles = w_tiles, g.per = sp.per;
            g.first = c0 == 0;
            g.part = direct ? nullptr : part + (kSmPartRows + 32) * (p.dp + 1);
            g.bias_part = nullptr, g.bias_out = nullptr, g.out = a.dh;
            SM_TRY((grad_pass<E, true>(p, g, sp.count, s)));
        }
    }
    if (a.dh != nullptr && !direct)
        SM_TRY(join<E>(p, part + (kSmPartRows + 32) * (p.dp + 1), sp.count, p.rows_pad, a.n,
                       a.scale, a.dh, nullptr, nullptr, s));
    return hipSuccess;
}

}  // namespace

SoftmaxPlan softmax_plan(int64_t classes, int64_t n, int32_t dim, int32_t dtype, bool grad) {
    SoftmaxPlan p{};
    p.dim = dim;
    p.parts = dtype == kDtypeBf16 ? 1 : 3;
    const int nd = (int)div_up(dim, 32);
    p.chunks = (int)div_up(nd, 8);
    p.nd = (int)div_up(nd, p.chunks);
    if (p.nd == 5 || p.nd == 7) ++p.nd;
    p.dp = 32 * p.nd * p.chunks;
    p.kd = (int)div_up(dim, 16);
    p.tile_elems = (int64_t)kSmTile * p.dp * p.parts;
    const int64_t forms = grad ? 2 : 1;
    const int64_t row_bytes = 2 * (int64_t)p.dp * p.parts * forms;
    p.piece = div_up(classes, kSmTile) * kSmTile;
    const int64_t most = kSmPieceBytes / row_bytes / kSmTile * kSmTile;
    if (p.piece > most) p.piece = most;
    p.rows_pad = n > 0 ? div_up(n, kSmTile) * kSmTile : kSmTile;
    size_t off = 0;
    auto take = [&](int64_t bytes) {
        const size_t o = off;
        off += ((size_t)bytes + 255) & ~(size_t)255;
        return o;
    };
    const int64_t h_bytes = 2 * (int64_t)p.dp * p.parts * p.rows_pad;
    const int64_t w_bytes = 2 * (int64_t)p.dp * p.parts * p.piece;
    p.hr = take(h_bytes);
    p.ht = take(grad ? h_bytes : 0);
    p.wr = take(w_bytes);
    p.wt = take(grad ? w_bytes : 0);
    p.yterm = take(4 * p.piece);
    p.xrow = take(grad ? 4 * p.rows_pad : 0);
    p.xlab = take(grad ? 4 * p.rows_pad : 0);
    p.xcw = take(grad ? 4 * p.rows_pad : 0);
    const int64_t rows = p.rows_pad > kSmPartRows ? p.rows_pad : kSmPartRows;
    p.part = take(grad ? 4 * ((kSmPartRows + 32) * (int64_t)(p.dp + 1) + rows * (int64_t)p.dp)
                       : 8 * rows);
    p.total = off;
    return p;
}

hipError_t launch_softmax_loss(const SoftmaxArgs& a, hipStream_t s) {
    if (a.n == 0) {
        if (a.loss_sum != nullptr) k_sm_sum<<<1, 1024, 0, s>>>(nullptr, 0, a.loss_sum);
        return hipGetLastError();
    }
    return a.dtype == kDtypeBf16 ? softmax_loss<bf16_t>(a, s) : softmax_loss<float>(a, s);
}

hipError_t launch_softmax_grad(const SoftmaxArgs& a, hipStream_t s) {
    return a.dtype == kDtypeBf16 ? softmax_grad<bf16_t>(a, s) : softmax_grad<float>(a, s);
}

}  // namespace huge
