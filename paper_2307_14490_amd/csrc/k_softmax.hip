// The calls of the exact softmax loss and its gradient (kernels: softmax.hpp).
#include "softmax.hpp"

namespace huge {

namespace {

// lse and loss of a row, LANES threads each: the splits are joined in an order that
// the sizes fix, and the label's logit is formed from the rows themselves.
template <typename E, int LANES>
__global__ __launch_bounds__(kBlock) void k_sm_loss(SoftmaxArgs a, const float2* __restrict__ part,
                                                    int splits, int64_t pad, int64_t first) {
    const int lane = threadIdx.x % LANES;
    const int64_t i = (first + blockIdx.x) * (kBlock / LANES) + threadIdx.x / LANES;
    if (i >= a.n) return;
    const int32_t y = a.labels[i];
    const float c = a.weight == nullptr ? 1.f : a.weight[i];
    float m = -INFINITY, sum = 0.f;
    for (int s = lane; s < splits; s += LANES) {
        const float2 p = part[(int64_t)s * pad + i];
        const float mm = fmaxf(m, p.x);
        sum = sum * exp_below(m, mm) + p.y * exp_below(p.x, mm);
        m = mm;
    }
#pragma unroll
    for (int off = 1; off < LANES; off <<= 1) {
        const float m2 = __shfl_xor(m, off), s2 = __shfl_xor(sum, off);
        const float mm = fmaxf(m, m2);
        sum = sum * exp_below(m, mm) + s2 * exp_below(m2, mm);
        m = mm;
    }
    // a NaN among the logits is in the sum, though no maximum
    const float lse = sum != sum ? sum : m == -INFINITY ? -INFINITY : m + logf(sum);
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
#pragma unroll 4
            for (int d = 4 * lane; d < a.dim; d += 4 * LANES)
                dot += dot4(load_cols(h, d, a.dim, a.vec), load_cols(w, d, a.dim, a.vec));
            const float below = lse - (group_sum<LANES>(dot) + b);
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

template <typename E>
hipError_t softmax_loss(SoftmaxArgs a, hipStream_t s) {
    const SoftmaxPlan p = softmax_plan(a.classes, a.n, a.dim, a.dtype, false);
    float2* part = reinterpret_cast<float2*>(a.ws + p.part);
    a.vec = fours(a.h, a.ld_h, sizeof(E)) && fours(a.w, a.ld_w, sizeof(E));
    constexpr int kN = 16 / sizeof(E);
    auto sixteen = [](const void* m, int64_t ld) {
        return (reinterpret_cast<uintptr_t>(m) & 15) == 0 && ld % kN == 0;
    };
    a.vec16 = a.dim % kN == 0 && sixteen(a.h, a.ld_h) && sixteen(a.w, a.ld_w);
    int64_t slots = 0, pad = p.rows_pad;
    const int few = few_blocks<E>(a.n, a.dim);
    if (few != 0) {
        pad = 16 * few;
        SM_TRY((few == 1   ? few_pass<E, 1>(a, part, &slots, s)
                : few == 2 ? few_pass<E, 2>(a, part, &slots, s)
                           : few_pass<E, 4>(a, part, &slots, s)));
    }
    // bf16 classes without a bias whose rows are whole operands are used as they lie:
    // no packing, for addresses per operand in a kernel that the vector units bind (1031
    // to 1131 us for 4096 x 1e6 x 128 against 960 to 1040).  Whole calls on one machine,
    // as they lie / through records: 4096 rows of that 1015 / 1104 us, 1024 rows 275 /
    // 390, 96 rows 82 / 207; 4096 x 50021 x 256 110 / 118.  The rows' share grows with
    // n: 8192 x 50021 x 128 119 / 123 us, x 512 397 / 382, 32768 x 50021 x 128 419 / 412,
    // x 512 1495 / 1386.
    const bool direct = few == 0 && sizeof(E) == 2 && a.bias == nullptr && a.vec16 &&
                        p.chunks == 1 && a.dim == p.dp;
    if (direct) {
        SM_TRY(pack<E>(p, a, 0, 0, 1, s));
        PassArgs l{};
        l.x = a.ws + p.h, l.forms = 1, l.first = true, l.lse_part = part;
        l.y_rows = static_cast<const bf16_t*>(a.w), l.ld = a.ld_w, l.classes = a.classes;
        l.x_tiles = p.rows_pad / kSmTile, l.y_tiles = div_up(a.classes, kSmTile);
        SM_TRY(lse_pass<E>(p, l, false, &slots, s));
    }
    for (int64_t c0 = 0; few == 0 && !direct && c0 < a.classes; c0 += p.piece) {
        const int64_t count = a.classes - c0 < p.piece ? a.classes - c0 : p.piece;
        SM_TRY(pack<E>(p, a, c0, count, 1, s));
        PassArgs l{};
        l.x = a.ws + p.h, l.y = a.ws + p.w, l.forms = 1;
        l.x_tiles = p.rows_pad / kSmTile, l.y_tiles = div_up(count, kSmTile);
        l.first = c0 == 0, l.lse_part = part;
        SM_TRY(lse_pass<E>(p, l, true, &slots, s));
    }
    // a wave a row until there are four for each SIMD, then 16 lanes.  16 / 64 lanes:
    // 256 rows behind 50021 classes of 128 fp32 columns 10.2 / 4.6 us, 1024 5.9 / 4.2, 4000 4.1
    // / 4.5 (of 384 bf16 columns 7.0 / 5.2), 16384 behind 1000 4.4 / 9.0, 100003 13.0 / 46.9
    if (a.n < 16 * kCus)
        k_sm_loss<E, 64><<<dim3((uint32_t)div_up(a.n, 4)), kBlock, 0, s>>>(a, part, (int)slots, pad, 0);
    else
        SM_TRY(in_launches(div_up(a.n, 16), [&](dim3 grid, int64_t first) {
            k_sm_loss<E, 16><<<grid, kBlock, 0, s>>>(a, part, (int)slots, pad, first);
        }));
    SM_TRY(hipGetLastError());
    if (a.loss_sum != nullptr) {
        k_sm_sum<<<1, 1024, 0, s>>>(a.loss, a.n, a.loss_sum);
        SM_TRY(hipGetLastError());
    }
    return hipSuccess;
}

}  // namespace

SoftmaxPlan softmax_plan(int64_t classes, int64_t n, int32_t dim, int32_t dtype, bool grad) {
    SoftmaxPlan p{};
    p.classes = classes;
    p.dim = dim;
    p.parts = dtype == kDtypeBf16 ? Kind<bf16_t>::kParts : Kind<float>::kParts;
    const int nd = (int)div_up(dim, 32);
    const int most = !grad ? 16 : p.parts == 2 && nd > 12 ? 8 : 12;
    p.chunks = (int)div_up(nd, nd > most && !grad ? 8 : most);
    p.nd = nd > most && !grad ? 8 : made_for((int)div_up(nd, p.chunks));
    p.dp = 32 * p.nd * p.chunks;
    p.kd = (int)div_up(dim, 16);
    const int64_t rec = record_bytes(p.dp / 16, p.parts, grad ? 2 : 1);
    p.piece = div_up(classes, kSmTile) * kSmTile;
    const int64_t fits = kSmPieceBytes / rec * kSmTile;
    if (p.piece > fits) p.piece = fits;
    p.rows_pad = n > 0 ? div_up(n, kSmTile) * kSmTile : kSmTile;
    size_t off = 0;
    auto take = [&](int64_t bytes) {
        const size_t o = off;
        off += ((size_t)bytes + 255) & ~(size_t)255;
        return o;
    };
    // losses of few rows pack nothing
    const bool packs = grad || (dtype == kDtypeBf16 ? few_blocks<bf16_t>(n, dim)
                                                    : few_blocks<float>(n, dim)) == 0;
    p.h = take(packs ? p.rows_pad / kSmTile * rec : 0);
    p.w = take(packs ? p.piece / kSmTile * rec : 0);
    const int64_t rows = p.rows_pad > kSmPartRows ? p.rows_pad : kSmPartRows;
    p.part = take(grad ? 4 * kSmPartRows * (int64_t)(p.dp + 1) : 8 * rows);
    p.row_part = take(grad ? 4 * rows * (int64_t)p.dp : 0);
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
    if (a.dh == nullptr && a.dw == nullptr && a.dbias == nullptr) return hipSuccess;
    return a.dtype == kDtypeBf16 ? softmax_grad<bf16_t>(a, s) : softmax_grad<float>(a, s);
}

}  // namespace huge
