// Log probabilities of given classes over a large vocabulary, with the entropy and the
// most likely classes, and their gradient, without the logits in memory.
//
// One pass over the logits (softmax.hpp) leaves a maximum, a sum of exponentials and
// their first moment per row and, where classes are to be found, the largest logit of
// each tile of 32 classes (16 for few rows): 1/32 of the logits' bytes.  The best `top`
// classes lie in the best `top` tiles, lowest first among equals, for a class outside
// of them has `top` tiles' largest before it.  So k_lp_select finds the best tiles of
// each row, kSlack more than that, for the matrix cores' logits are a rounding away from the ones
// that decide, and k_lp_top forms the logits of their classes again in fp64, in which
// products of bf16 or fp32 numbers are exact, and orders those.
//
// 4096 x 1e6 x 128 bf16, ten best: the pass 1257 to 1380 us by the clock (0.76 to 0.83 PFLOP/s;
// the loss, which needs no moment and no tile's largest, takes 960 to 1040), the search 107
// (0.5 GB of largest logits at 4.8 TB/s), the best classes 92 (470 MB of table rows).  The pass
// is bound by the vector units: 16 exponentials of 16 clocks and about 55 other instructions
// of 4 for a tile of 32 x 32, where its products take 256; they are busy 74% of the time.
// One row over 1e6 x 128 in 8 bits: 30 us (132 MB at 4.4 TB/s), 11 and 9.  With more than 64 rows a
// table in 8 bits is widened into records in every call, 115 to 127 us for this one: 128 rows 240 us
// in all, in bf16 120; 4096 rows 1652 and 1618.
#include "softmax.hpp"

namespace huge {

namespace {

typedef unsigned long long u64;

constexpr int kSlack = 4;                          // tiles looked at beyond `top`
constexpr int kTopThreads = 256;
constexpr int64_t kBestBytes = (int64_t)1 << 30;   // tile maxima and lists at a time
constexpr int kThirdsFrom = 3;                     // blocks of 16 fp32 rows that go in thirds
constexpr int64_t kBestRows = 8192;                // rows that have room for any piece
constexpr int64_t kListRows = 32768;               // rows times splits of k_lp_select
constexpr int kMostSplits = 64;
constexpr int kTopLds = 80 * 1024;
constexpr int64_t kMostRows = (int64_t)1 << 22;    // rows at a time: a workgroup each

// A tile's key: its largest logit, then the lower tile.  0 is below all keys.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ u64 tile_key(uint32_t order, uint32_t tile) {
    return (u64)order << 32 | (uint32_t)~tile;
}
__device__ __forceinline__ int64_t key_tile(u64 key) { return (int64_t)(uint32_t)~(uint32_t)key; }

// Dot product of a row h (fp64 in LDS) with a class's row, by the LANES threads of a group.
template <typename E, bool CODES, int LANES>
__device__ __forceinline__ double dot64(const SoftmaxArgs& a, const double* h, int64_t cls, int lane) {
    double s = 0.0;
#pragma unroll 4
    for (int d = 4 * lane; d < a.dim; d += 4 * LANES) {
        float4 v;
        if constexpr (CODES)
            v = load_code_cols(static_cast<const uint8_t*>(a.w) + cls * a.ld_w,
                               a.w_scales + cls * a.ld_scales, d, a.dim, a.vec);
        else
            v = load_cols(static_cast<const E*>(a.w) + cls * a.ld_w, d, a.dim, a.vec);
        s = fma(h[d], (double)v.x, s);
        s = fma(h[d + 1], (double)v.y, s);
        s = fma(h[d + 2], (double)v.z, s);
        s = fma(h[d + 3], (double)v.w, s);
    }
#pragma unroll
    for (int off = 1; off < LANES; off <<= 1) s += __shfl_xor(s, off);
    return s;
}

// ---------------------------------------------------------------------------
// lse, entropy and the label's log probability of a row, LANES threads each
// ---------------------------------------------------------------------------
// Over the LANES threads of a row, in the same order always; a workgroup's four waves meet
// in s, and all of its threads call.
template <int LANES, typename T>
__device__ __forceinline__ T row_add(T v, double* s) {
#pragma unroll
    for (int off = 1; off < (LANES < 64 ? LANES : 64); off <<= 1) v += __shfl_xor(v, off);
    if constexpr (LANES > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = (double)v;
        __syncthreads();
        v = (T)s[0] + (T)s[1] + (T)s[2] + (T)s[3];
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float row_max(float v, double* s) {
#pragma unroll
    for (int off = 1; off < (LANES < 64 ? LANES : 64); off <<= 1) v = fmaxf(v, __shfl_xor(v, off));
    if constexpr (LANES > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = (double)v;
        __syncthreads();
        v = fmaxf(fmaxf((float)s[0], (float)s[1]), fmaxf((float)s[2], (float)s[3]));
    }
    return v;
}

// What the pass over the logits leaves: `slots` entries of each row.
struct Parts {
    const float4* p;
    int64_t of_slot, of_row;  // strides
    int32_t slots;
    __device__ __forceinline__ float4 at(int64_t row, int64_t slot) const {
        return p[slot * of_slot + row * of_row];
    }
};

// Row i, by LANES threads.  s_join: of a workgroup of four waves where LANES is all of it.
template <typename E, bool CODES, int LANES>
__device__ __forceinline__ void answer_row(const SoftmaxArgs& a, const Parts& part, int64_t i,
                                           int lane, double* s_join) {
    // the top of all slots first, then their sums from it: one exponential a slot, none of
    // which waits for another
    float top = kLeast;
#pragma unroll 8
    for (int k = lane; k < part.slots; k += LANES) top = fmaxf(top, part.at(i, k).x);
    top = row_max<LANES>(top, s_join);
    float sum = 0.f, first = 0.f;
#pragma unroll 8
    for (int k = lane; k < part.slots; k += LANES) {
        const float4 p = part.at(i, k);
        const Stats s = raise({p.x, p.y, p.z}, top);
        sum += s.sum;
        first += s.first;
    }
    sum = row_add<LANES>(sum, s_join), first = row_add<LANES>(first, s_join);
    const float logs = logf(sum);
    const float lse = sum == 0.f ? -INFINITY : top + logs;
    float entropy = sum == 0.f ? 0.f : logs - 0.69314718055994531f * (first / sum);
    entropy = entropy < 0.f ? 0.f : entropy;  // rounding alone takes it below 0
    float logp = 0.f;
    if (a.labels != nullptr) {
        const int32_t y = a.labels[i];
        if (y < -1 || y >= a.classes) {
            logp = NAN;
            if (lane == 0) set_status(a.status, -2);
        } else if (y >= 0) {
            const float b = a.bias == nullptr ? 0.f : a.bias[y];
            if (b < kLeast) {
                logp = -INFINITY;
            } else {
                const E* h = static_cast<const E*>(a.h) + i * a.ld_h;
                double dot = 0.0;
#pragma unroll 4
                for (int d = 4 * lane; d < a.dim; d += 4 * LANES) {
                    const float4 u = load_cols(h, d, a.dim, a.vec_h);
                    float4 v;
                    if constexpr (CODES)
                        v = load_code_cols(static_cast<const uint8_t*>(a.w) + y * a.ld_w,
                                           a.w_scales + y * a.ld_scales, d, a.dim, a.vec);
                    else
                        v = load_cols(static_cast<const E*>(a.w) + y * a.ld_w, d, a.dim, a.vec);
                    dot = fma((double)u.x, (double)v.x, dot);
                    dot = fma((double)u.y, (double)v.y, dot);
                    dot = fma((double)u.z, (double)v.z, dot);
                    dot = fma((double)u.w, (double)v.w, dot);
                }
                dot = row_add<LANES>(dot, s_join);
                logp = (float)(dot + (double)b - (double)lse);
                logp = logp > 0.f ? 0.f : logp;  // as above
            }
        }
    }
    if (lane == 0) {
        a.lse[i] = lse;
        if (a.entropy != nullptr) a.entropy[i] = entropy;
        if (a.logp != nullptr) a.logp[i] = logp;
    }
}

template <typename E, bool CODES, int LANES>
__global__ __launch_bounds__(kBlock) void k_lp_rows(SoftmaxArgs a, Parts part, int64_t rows,
                                                    int64_t first) {
    __shared__ double s_join[4];
    const int64_t i = (first + blockIdx.x) * (kBlock / LANES) + threadIdx.x / LANES;
    if (i < rows) answer_row<E, CODES, LANES>(a, part, i, threadIdx.x % LANES, s_join);
}

// ---------------------------------------------------------------------------
// The best tiles of each row
// ---------------------------------------------------------------------------
// A workgroup takes RW rows and a split of the tiles.  What is above a row's bar goes to
// its list in LDS, whose order does not matter.  The bar: each slot of the pass over the
// logits has left its largest logit, of another tile each, so that the best `keep` of all
// tiles are at or above the keep-th largest of those (of some threads' largest of them).
// A list that overflows all the same is built again in rounds of four tiles a thread: one that
// the next round could overfill is cut to its best `keep`, the last of which is the new
// bar.  Tiles come in rising order from round to round, so that an equal one of a later
// round is not better.
//
// Without the bar every list filled and was cut in each round's turn: 4096 x 31250 tiles 375 us,
// 107 with it; the 62500 tiles of one row 47 us, 11.
//
// There is none where the bar's `keep` = top + 4 values are not to be had: from as many threads of
// a row (32, of few rows 64: top above 28, 60) and slots of the pass (about kSmPartRows / rows:
// rows (top + 4) above 131072 at a time).  Lists then go in rounds.  bf16, D = 128: 4096 x 1e6, 28 best
// 134 us, 29 best 576, 64 best 697; 250000 classes, ten best of 8192 rows 71, of 9376 467; of 16384 rows
// three best 129, ten best 515.
constexpr int kSelectThreads = 1024;
constexpr int kSelectKeys = 10496;
template <int RW>
struct Select {
    static constexpr int kSubs = kSelectThreads / RW;   // threads of a row
    static constexpr int kRound = 4 * kSubs;            // tiles of a round
    static constexpr int kRoom = kSelectKeys / RW;      // keys of a row's list
    static_assert(kRoom >= kRound + kMostTop + kSlack, "a round fits behind a cut list");
};

// Cuts each list to its best `keep`, in order.
template <int RW>
__device__ __forceinline__ void cut_lists(u64* keys, int* count, uint32_t* least, int keep) {
    using S = Select<RW>;
    constexpr int kOwn = (S::kRoom + S::kSubs - 1) / S::kSubs;
    const int row = threadIdx.x / S::kSubs, lane = threadIdx.x % S::kSubs;
    u64* list = keys + row * S::kRoom;
    const int n = count[row];
    u64 own[kOwn];
    int rank[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        own[k] = lane + k * S::kSubs < n ? list[lane + k * S::kSubs] : 0;
        rank[k] = 0;
    }
    for (int j = 0; j < n; ++j) {
        const u64 key = list[j];
#pragma unroll
        for (int k = 0; k < kOwn; ++k) rank[k] += key > own[k] ? 1 : 0;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
        if (own[k] != 0 && rank[k] < keep) {
            list[rank[k]] = own[k];
            if (rank[k] == keep - 1) least[row] = (uint32_t)(own[k] >> 32);
        }
    if (lane == 0) count[row] = n < keep ? n : keep;
    __syncthreads();
}

// The last row of workgroups of a call's last search forms the rows' own results beside it.
template <typename E, bool CODES, int RW>
__global__ __launch_bounds__(kSelectThreads) void k_lp_select(SoftmaxArgs a,
                                                              const float* __restrict__ best,
                                                              int64_t ld, int64_t rows,
                                                              int64_t tiles, int64_t tile0,
                                                              int64_t per, int splits, int keep,
                                                              Parts part, u64* __restrict__ lists) {
    using S = Select<RW>;
    if ((int)blockIdx.y == splits) {
        const int64_t i = (int64_t)blockIdx.x * RW + threadIdx.x / S::kSubs;
        if (i < rows) answer_row<E, CODES, S::kSubs>(a, part, i, threadIdx.x % S::kSubs, nullptr);
        return;
    }
    extern __shared__ __align__(16) uint8_t lds[];
    u64* keys = reinterpret_cast<u64*>(lds);  // [RW][kRoom]
    __shared__ int count[RW];
    __shared__ uint32_t least[RW];
    __shared__ bool over;
    const int r = threadIdx.x % RW, sub = threadIdx.x / RW;
    const int64_t row = (int64_t)blockIdx.x * RW + r;
    const bool in = row < rows;
    // a tile whose classes are all out has kFloor
    if (threadIdx.x < RW) count[threadIdx.x] = 0, least[threadIdx.x] = ordered(kLeast);
    if (threadIdx.x == 0) over = false;
    const int64_t t0 = (int64_t)blockIdx.y * per;
    const int64_t t1 = t0 + per < tiles ? t0 + per : tiles;
    constexpr int kDeep = 8;
    auto load = [&](int64_t at, float* v, int n) {
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            if (k >= n) break;
            const int64_t t = at + sub + k * S::kSubs;
            v[k] = in && t < t1 ? best[t * ld + row] : NAN;
        }
    };
    float now[kDeep], next[kDeep];
    load(t0, now, kDeep);
    if (keep <= S::kSubs) {
        float v = -INFINITY;
        if (in)
#pragma unroll 8
            for (int k = sub; k < part.slots; k += S::kSubs) v = fmaxf(v, part.at(row, k).w);
        uint32_t* of_row = reinterpret_cast<uint32_t*>(lds);  // [sub][row]
        const uint32_t own = v > kLeast ? ordered(v) : 0;
        of_row[threadIdx.x] = own;
        __syncthreads();
        int rank = 0;
#pragma unroll 8
        for (int k = 0; k < S::kSubs; ++k) {
            const uint32_t o = of_row[k * RW + r];
            rank += o > own || (o == own && k < sub) ? 1 : 0;
        }
        if (rank == keep - 1 && own != 0) least[r] = own - 1;
    }
    __syncthreads();
    const uint32_t bar = least[r];
    for (int64_t at = t0; at < t1; at += kDeep * S::kSubs) {
        load(at + kDeep * S::kSubs, next, kDeep);
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const uint32_t o = ordered(now[k]);
            if (now[k] == now[k] && o > bar) {
                const int slot = atomicAdd(&count[r], 1);
                if (slot < S::kRoom)
                    keys[r * S::kRoom + slot] =
                        tile_key(o, (uint32_t)(tile0 + at + sub + k * S::kSubs));
                else
                    over = true;
            }
            now[k] = next[k];
        }
    }
    __syncthreads();
    if (over) {
        __syncthreads();
        if (threadIdx.x < RW) count[threadIdx.x] = 0;
        __syncthreads();
        for (int64_t at = t0; at < t1; at += S::kRound) {
            load(at, now, 4);
            const uint32_t above = least[r];
            bool full = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t o = ordered(now[k]);
                if (now[k] == now[k] && o > above) {
                    const int slot = atomicAdd(&count[r], 1);
                    keys[r * S::kRoom + slot] =
                        tile_key(o, (uint32_t)(tile0 + at + sub + k * S::kSubs));
                    full |= slot >= S::kRoom - S::kRound - 1;
                }
            }
            if (__syncthreads_or(full)) cut_lists<RW>(keys, count, least, keep);
        }
    }
    cut_lists<RW>(keys, count, least, keep);
    for (int j = threadIdx.x; j < RW * keep; j += kSelectThreads) {
        const int k = j / keep;
        const int64_t out = (int64_t)blockIdx.x * RW + k;
        if (out < rows)
            lists[(out * splits + blockIdx.y) * keep + j % keep] =
                j % keep < count[k] ? keys[k * S::kRoom + j % keep] : 0;
    }
}

// The best `keep` of the n keys of `splits` lists in LDS to `out` (LDS too), in order; 0
// behind the last.  A key below the last of a full list is not one of them.  `left` (LDS)
// has room for n.
template <int THREADS>
__device__ __forceinline__ void best_keys(const u64* keys, int n, int keep, u64* left, u64* out) {
    __shared__ u64 s_bar;
    __shared__ int s_count;
    if (threadIdx.x == 0) s_bar = 0, s_count = 0;
    for (int e = threadIdx.x; e < keep; e += THREADS) out[e] = 0;
    __syncthreads();
    for (int e = keep - 1 + keep * threadIdx.x; e < n; e += keep * THREADS)
        if (keys[e] != 0) atomicMax(&s_bar, keys[e]);
    __syncthreads();
    const u64 bar = s_bar;
    for (int e = threadIdx.x; e < n; e += THREADS)
        if (keys[e] != 0 && keys[e] >= bar) left[atomicAdd(&s_count, 1)] = keys[e];
    __syncthreads();
    const int m = s_count;
    for (int e = threadIdx.x; e < m; e += THREADS) {
        const u64 own = left[e];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < m; ++j) rank += left[j] > own ? 1 : 0;
        if (rank < keep) out[rank] = own;
    }
    __syncthreads();
}

// A row's lists of `splits`, and of the pieces of the vocabulary before, into one.
__global__ __launch_bounds__(kTopThreads) void k_lp_merge(const u64* __restrict__ lists, int splits,
                                                          int keep, bool first,
                                                          u64* __restrict__ running) {
    extern __shared__ __align__(16) uint8_t lds[];
    const int64_t row = blockIdx.x;
    const int n = splits * keep;
    u64* s_out = reinterpret_cast<u64*>(lds);
    u64* s_keys = s_out + keep;  // the lists, twice
    for (int e = threadIdx.x; e < n; e += kTopThreads) s_keys[e] = lists[row * n + e];
    if (!first)
        for (int e = threadIdx.x; e < keep; e += kTopThreads) s_keys[n + e] = running[row * keep + e];
    __syncthreads();
    best_keys<kTopThreads>(s_keys, first ? n : n + keep, keep, s_keys + n + keep, s_out);
    for (int e = threadIdx.x; e < keep; e += kTopThreads) running[row * keep + e] = s_out[e];
}

// The best classes of a row among those of its best tiles of G.  Eight threads form a
// class's logit; what is then below the top-th largest of the tiles' largest is dropped, and
// the few others are ranked by counting.  Bound by the rows that it reads; for few rows by
// its four steps, each behind the last (9 us, by four times the threads).
template <typename E, bool CODES, int G, int THREADS>
__global__ __launch_bounds__(THREADS) void k_lp_top(SoftmaxArgs a, const u64* __restrict__ lists,
                                                    int splits, int keep) {
    constexpr int kLanes = 8, kAtOnce = THREADS / kLanes;
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ double s_bar;
    __shared__ int s_count;
    const int n = splits * keep, m = keep * G;
    double* s_h = reinterpret_cast<double*>(lds);             // the row
    u64* s_best = reinterpret_cast<u64*>(s_h + a.dim);        // its best tiles
    double* s_most = reinterpret_cast<double*>(s_best + keep);  // the largest logit of each
    double* s_x = s_most + keep;                              // their classes' logits
    int* s_left = reinterpret_cast<int*>(s_x + m);            // those that may be wanted
    u64* s_keys = reinterpret_cast<u64*>(s_x);                // before: the lists, twice
    const int64_t row = blockIdx.x;
    const float lse = a.lse[row];
    int32_t* ids = a.ids + row * a.top;
    float* logp = a.top_logp + row * a.top;
    if (!(lse > -INFINITY && lse < INFINITY)) {  // no class, or no number
        for (int k = threadIdx.x; k < a.top; k += THREADS) {
            ids[k] = -1;
            logp[k] = lse == -INFINITY ? -INFINITY : NAN;
        }
        return;
    }
    for (int e = threadIdx.x; e < n; e += THREADS) s_keys[e] = lists[row * n + e];
    const E* h = static_cast<const E*>(a.h) + row * a.ld_h;
    for (int d = 4 * threadIdx.x; d < a.dim; d += 4 * THREADS) {
        const float4 v = load_cols(h, d, a.dim, a.vec_h);
        s_h[d] = v.x, s_h[d + 1] = v.y, s_h[d + 2] = v.z, s_h[d + 3] = v.w;
    }
    if (threadIdx.x == 0) s_bar = -INFINITY, s_count = 0;
    __syncthreads();
    best_keys<THREADS>(s_keys, n, keep, s_keys + n, s_best);
    auto class_of = [&](int e) { return key_tile(s_best[e / G]) * G + e % G; };
    const int lane = threadIdx.x % kLanes;
    for (int e = threadIdx.x / kLanes; e < m; e += kAtOnce) {
        const int64_t cls = class_of(e);
        double x = -INFINITY;
        if (s_best[e / G] != 0 && cls < a.classes) {
            const float b = a.bias == nullptr ? 0.f : a.bias[cls];
            if (!(b < kLeast)) x = dot64<E, CODES, kLanes>(a, s_h, cls, lane) + (double)b;
        }
        if (lane == 0) s_x[e] = x;
    }
    __syncthreads();
    // at least `top` classes are at or above the top-th largest of the tiles' largest
    if (threadIdx.x < keep) {
        double v = -INFINITY;
#pragma unroll 8
        for (int e = 0; e < G; ++e) v = fmax(v, s_x[threadIdx.x * G + e]);
        s_most[threadIdx.x] = v;
    }
    __syncthreads();
    if (threadIdx.x < keep) {
        const double own = s_most[threadIdx.x];
        int rank = 0;
        for (int k = 0; k < keep; ++k)
            rank += s_most[k] > own || (s_most[k] == own && k < (int)threadIdx.x) ? 1 : 0;
        if (rank == a.top - 1) s_bar = own;
    }
    __syncthreads();
    const double bar = s_bar;
    for (int e = threadIdx.x; e < m; e += THREADS)
        if (s_x[e] > -INFINITY && s_x[e] >= bar) s_left[atomicAdd(&s_count, 1)] = e;
    __syncthreads();
    const int c = s_count;
    for (int k = threadIdx.x; k < c; k += THREADS) {
        const double x = s_x[s_left[k]];
        const int64_t cls = class_of(s_left[k]);
        int rank = 0;
        for (int j = 0; j < c && rank < a.top; ++j) {
            const double y = s_x[s_left[j]];
            rank += y > x || (y == x && class_of(s_left[j]) < cls) ? 1 : 0;
        }
        if (rank < a.top) {
            const float l = (float)(x - (double)lse);
            ids[rank] = (int32_t)cls;
            logp[rank] = l > 0.f ? 0.f : l;
        }
    }
    for (int k = c + threadIdx.x; k < a.top; k += THREADS) ids[k] = -1, logp[k] = -INFINITY;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
int64_t round_down(int64_t v, int64_t to) { return v / to * to; }

// Splits of a select of `rows` padded rows over `tiles`: about two workgroups a CU, each
// with a few rounds.
int select_splits(int64_t rows, int64_t tiles, int rw) {
    const int64_t blocks = div_up(rows, rw);
    int64_t s = 512 / blocks;
    const int64_t most = tiles / (4 * 4 * (kSelectThreads / rw));
    if (s > most) s = most;
    if (s > kMostSplits) s = kMostSplits;
    if (s > kListRows / rows) s = kListRows / rows;
    return (int)(s < 1 ? 1 : s);
}

// last: with the rows' own results.
template <typename E, bool CODES, int RW>
hipError_t select(const SoftmaxArgs& a, const float* best, int64_t ld, int64_t rows, int64_t tiles,
                  int64_t tile0, int splits, int keep, const Parts& part, u64* lists, bool last,
                  hipStream_t s) {
    constexpr auto* kKernel = &k_lp_select<E, CODES, RW>;
    SM_TRY(allow_lds<kKernel>(kSelectKeys * 8));
    const dim3 grid((uint32_t)div_up(rows, RW), (uint32_t)(splits + (last ? 1 : 0)));
    kKernel<<<grid, kSelectThreads, kSelectKeys * 8, s>>>(a, best, ld, rows, tiles, tile0,
                                                          div_up(tiles, splits), splits, keep, part,
                                                          lists);
    return hipGetLastError();
}

hipError_t merge(const u64* lists, int splits, int keep, bool first, u64* running, int64_t rows,
                 hipStream_t s) {
    const int lds = 8 * (2 * (splits + 1) + 1) * keep;
    if (lds > 64 * 1024) SM_TRY(allow_lds<&k_lp_merge>(kTopLds));
    k_lp_merge<<<dim3((uint32_t)rows), kTopThreads, lds, s>>>(lists, splits, keep, first, running);
    return hipGetLastError();
}

// What is left behind the passes: the rows' own results where nothing is to be found, or
// the best classes.
template <typename E, bool CODES, int G>
hipError_t finish(const SoftmaxArgs& a, const AnswerPlan& p, const Parts& part, int64_t rows,
                  int splits, const u64* lists, hipStream_t s) {
    if (a.top == 0) {
        if (rows < kCus)
            k_lp_rows<E, CODES, 256><<<dim3((uint32_t)rows), kBlock, 0, s>>>(a, part, rows, 0);
        else if (rows < 16 * kCus)
            k_lp_rows<E, CODES, 64><<<dim3((uint32_t)div_up(rows, 4)), kBlock, 0, s>>>(a, part, rows, 0);
        else if (rows < 128 * kCus)
            k_lp_rows<E, CODES, 16><<<dim3((uint32_t)div_up(rows, 16)), kBlock, 0, s>>>(a, part, rows, 0);
        else  // fewer waves, each with more loads in flight: 100003 x 1000 x 128 bf16 12.9 us, 18.5 with 16
            SM_TRY(in_launches(div_up(rows, 32), [&](dim3 grid, int64_t first) {
                k_lp_rows<E, CODES, 8><<<grid, kBlock, 0, s>>>(a, part, rows, first);
            }));
        return hipGetLastError();
    }
    const int lists_ = 2 * splits * p.keep, logits = p.keep * G + (p.keep * G + 1) / 2;
    const int lds = 8 * (a.dim + 2 * p.keep + (lists_ > logits ? lists_ : logits));
    if (rows < kCus) {
        constexpr auto* kKernel = &k_lp_top<E, CODES, G, 1024>;
        if (lds > 64 * 1024) SM_TRY(allow_lds<kKernel>(kTopLds));
        kKernel<<<dim3((uint32_t)rows), 1024, lds, s>>>(a, lists, splits, p.keep);
    } else {
        constexpr auto* kKernel = &k_lp_top<E, CODES, G, kTopThreads>;
        if (lds > 64 * 1024) SM_TRY(allow_lds<kKernel>(kTopLds));
        kKernel<<<dim3((uint32_t)rows), kTopThreads, lds, s>>>(a, lists, splits, p.keep);
    }
    return hipGetLastError();
}

// The same arguments for rows r0 .. of them.
template <typename E>
SoftmaxArgs rows_from(SoftmaxArgs a, int64_t r0) {
    a.h = static_cast<const E*>(a.h) + r0 * a.ld_h;
    if (a.labels != nullptr) a.labels += r0;
    a.lse += r0;
    if (a.entropy != nullptr) a.entropy += r0;
    if (a.logp != nullptr) a.logp += r0;
    if (a.top > 0) a.ids += r0 * a.top, a.top_logp += r0 * a.top;
    return a;
}

// ... and for `count` classes from c0 on.
template <typename E, bool CODES>
SoftmaxArgs classes_from(SoftmaxArgs a, int64_t c0, int64_t count) {
    if constexpr (CODES) {
        a.w = static_cast<const uint8_t*>(a.w) + c0 * a.ld_w;
        a.w_scales += c0 * a.ld_scales;
    } else {
        a.w = static_cast<const E*>(a.w) + c0 * a.ld_w;
    }
    if (a.bias != nullptr) a.bias += c0;
    a.classes = count;
    return a;
}

template <typename E, bool CODES>
hipError_t log_probs(SoftmaxArgs a, hipStream_t s) {
    const AnswerPlan p = answer_plan(a.classes, a.n, a.dim, a.dtype, CODES, a.top);
    float4* part = reinterpret_cast<float4*>(a.ws + p.part);
    float* best = a.top > 0 ? reinterpret_cast<float*>(a.ws + p.best) : nullptr;
    u64* lists = reinterpret_cast<u64*>(a.ws + p.lists);
    u64* running = reinterpret_cast<u64*>(a.ws + p.running);
    constexpr int kN = CODES ? 16 : 16 / (int)sizeof(E), kNh = 16 / sizeof(E);
    auto sixteen = [](const void* m, int64_t ld, int n) {
        return (reinterpret_cast<uintptr_t>(m) & 15) == 0 && ld % n == 0;
    };
    a.vec_h = fours(a.h, a.ld_h, sizeof(E));
    a.vec = fours(a.w, a.ld_w, CODES ? 1 : sizeof(E));
    a.vec16 = a.dim % kN == 0 && sixteen(a.w, a.ld_w, kN);
    if constexpr (!CODES) {
        // the few rows' kernel reads both alike
        a.vec16 = a.vec16 && sixteen(a.h, a.ld_h, kNh);
    }
    const int64_t all = div_up(a.classes, p.group), piece = p.piece / p.group;
    if (p.few != 0) {
        SoftmaxArgs f = a;
        if constexpr (!CODES) f.vec = a.vec && a.vec_h;
        const int64_t pad = 16 * p.few;
        const bool pieces = piece < all;
        // calls with(blocks of 16 rows, thirds), as types
        auto dispatch = [&](auto with) {
            auto of = [&](auto nb) {
                if constexpr (sizeof(E) == 4 && decltype(nb)::value >= kThirdsFrom)
                    if (p.thirds) return with(nb, std::true_type{});
                return with(nb, std::false_type{});
            };
            return p.few == 1   ? of(std::integral_constant<int, 1>{})
                   : p.few == 2 ? of(std::integral_constant<int, 2>{})
                   : p.few == 3 ? of(std::integral_constant<int, 3>{})
                                : of(std::integral_constant<int, 4>{});
        };
        int64_t slots = 0, all_slots = 0;
        for (int64_t t0 = 0; t0 < all; t0 += piece) {
            const int64_t left = a.classes - t0 * 16, count = left < piece * 16 ? left : piece * 16;
            all_slots += dispatch([&](auto nb, auto thirds) {
                return few_grid<E, decltype(nb)::value, true, CODES, decltype(thirds)::value>(count,
                                                                                            a.dim);
            });
        }
        int splits = 1;
        for (int64_t t0 = 0; t0 < all; t0 += piece) {
            const int64_t tiles = all - t0 < piece ? all - t0 : piece, c0 = t0 * 16;
            const int64_t count = a.classes - c0 < tiles * 16 ? a.classes - c0 : tiles * 16;
            const SoftmaxArgs q = classes_from<E, CODES>(f, c0, count);
            int64_t more = 0;
            SM_TRY(dispatch([&](auto nb, auto thirds) {
                return few_pass<E, decltype(nb)::value, true, CODES, decltype(thirds)::value>(
                    q, part, &more, s, best, all_slots, slots);
            }));
            slots += more;
            if (a.top == 0) continue;
            splits = select_splits(pad, tiles, 16);
            const Parts now{part, 1, all_slots, (int32_t)slots};
            SM_TRY((select<E, CODES, 16>(a, best, pad, a.n, tiles, t0, splits, p.keep, now, lists,
                                         t0 + tiles == all, s)));
            if (!pieces) continue;
            SM_TRY(merge(lists, splits, p.keep, t0 == 0, running, a.n, s));
        }
        return finish<E, CODES, 16>(a, p, Parts{part, 1, all_slots, (int32_t)all_slots}, a.n,
                                    pieces ? 1 : splits, pieces ? running : lists, s);
    }
    // bf16 classes without a bias are used as they lie, as in the loss
    const bool direct = !CODES && sizeof(E) == 2 && a.bias == nullptr && a.vec16 &&
                        p.sm.chunks == 1 && a.dim == p.sm.dp;
    const bool pieces = piece < all;
    SoftmaxPlan sm = p.sm;
    sm.piece = p.piece;
    const int64_t rec = record_bytes(sm.dp / 16, sm.parts, 1);
    // ... and so are bf16 rows of whole operands, which a wave reads once
    const bool x_direct = sizeof(E) == 2 && p.sm.chunks == 1 && a.dim == p.sm.dp &&
                          sixteen(a.h, a.ld_h, kNh);
    if (direct && !x_direct) SM_TRY((pack<E, true, CODES>(sm, a, 0, 0, 1, s)));  // the rows
    for (int64_t r0 = 0; r0 < a.n; r0 += p.rows) {
        const int64_t rows = a.n - r0 < p.rows ? a.n - r0 : p.rows;
        const SoftmaxArgs q = rows_from<E>(a, r0);
        int64_t slots = 0;
        int splits = 1;
        PassArgs l{};
        l.x = a.ws + p.sm.h + r0 / kSmTile * rec, l.forms = 1, l.stat_part = part;
        if (x_direct) l.x_direct = static_cast<const bf16_t*>(q.h), l.x_ld = a.ld_h, l.x_count = rows;
        l.x_tiles = div_up(rows, kSmTile);
        const int64_t pad = l.x_tiles * kSmTile;
        l.best = best, l.best_ld = pad;
        for (int64_t t0 = 0; t0 < all; t0 += piece) {
            const int64_t tiles = all - t0 < piece ? all - t0 : piece, c0 = t0 * kSmTile;
            const int64_t count = a.classes - c0 < tiles * kSmTile ? a.classes - c0 : tiles * kSmTile;
            if (!direct && (pieces || r0 == 0))
                SM_TRY((pack<E, true, CODES>(sm, a, c0, count, 1, s, !x_direct)));
            if (direct)
                l.y_rows = static_cast<const bf16_t*>(a.w) + c0 * a.ld_w, l.ld = a.ld_w, l.classes = count;
            else
                l.y = a.ws + p.sm.w;
            l.y_tiles = tiles, l.first = t0 == 0;
            SM_TRY((lse_pass<E, true>(sm, l, true, &slots, s)));
            if (a.top == 0) continue;
            splits = select_splits(pad, tiles, 32);
            SM_TRY((select<E, CODES, 32>(q, best, pad, rows, tiles, t0, splits, p.keep,
                                         Parts{part, pad, 1, (int32_t)slots}, lists,
                                         t0 + tiles == all, s)));
            if (!pieces) continue;
            SM_TRY(merge(lists, splits, p.keep, t0 == 0, running, rows, s));
        }
        SM_TRY((finish<E, CODES, 32>(q, p, Parts{part, pad, 1, (int32_t)slots}, rows,
                                     pieces ? 1 : splits, pieces ? running : lists, s)));
    }
    return hipSuccess;
}

}  // namespace

AnswerPlan answer_plan(int64_t classes, int64_t n, int32_t dim, int32_t dtype, bool codes,
                       int32_t top) {
    AnswerPlan p{};
    const bool bf16 = dtype == kDtypeBf16;
    p.sm = softmax_plan(classes, n, dim, dtype, false);
    const int64_t blocks = div_up(n, 16);
    if (blocks <= 4) {
        p.thirds = !bf16 && blocks >= kThirdsFrom &&
                   few_kb<float, false, true>(dim) * blocks * 1024 <= kFewLds<float>;
        const int64_t kb = p.thirds ? 0 : codes ? few_kb<bf16_t, true>(dim)
                           : bf16 ? few_kb<bf16_t, false>(dim) : few_kb<float, false>(dim);
        if (kb * blocks * 1024 <= (bf16 ? kFewLds<bf16_t> : kFewLds<float>)) p.few = (int32_t)blocks;
    }
    p.group = p.few != 0 ? 16 : kSmTile;
    const int64_t all = div_up(classes, p.group);
    const int64_t pad = p.few != 0 ? 16 * p.few : p.sm.rows_pad;
    const int64_t rec = record_bytes(p.sm.dp / 16, p.sm.parts, 1);
    p.keep = (int32_t)(all < top + kSlack ? all : top + kSlack);
    int64_t piece = all;  // tiles at a time
    p.rows = pad;         // rows at a time
    if (p.few == 0 && piece > kSmPieceBytes / rec) piece = kSmPieceBytes / rec;
    if (top > 0) {
        // the same piece for every number of rows, so that fewer never need more memory
        const int64_t least = p.few != 0 ? pad : kBestRows;
        const int64_t lists = 16 * (int64_t)p.keep;  // of a row, and those of earlier pieces
        const int64_t fits = (kBestBytes / least - lists) / 4;
        if (piece > fits) piece = fits;
        int64_t most = round_down(kBestBytes / (4 * piece + lists), kSmTile);
        if (most > kMostRows) most = kMostRows;
        if (p.few == 0 && p.rows > most) p.rows = most;
    }
    p.piece = piece * p.group;
    size_t off = 0;
    auto take = [&](int64_t bytes) {
        const size_t o = off;
        off += ((size_t)bytes + 255) & ~(size_t)255;
        return o;
    };
    p.sm.h = take(p.few != 0 ? 0 : p.sm.rows_pad / kSmTile * rec);
    p.sm.w = take(p.few != 0 ? 0 : piece * rec);
    const int64_t slots = p.few != 0 ? 2048 * div_up(all, piece) * pad : 0;
    const int64_t parts = p.rows > kSmPartRows ? p.rows : kSmPartRows;
    p.part = take(16 * (slots > parts ? slots : parts));
    if (top > 0) {
        p.best = take(4 * p.rows * piece);
        p.lists = take(8 * (p.rows > kListRows ? p.rows : kListRows) * p.keep);
        p.running = take(piece < all ? 8 * p.rows * p.keep : 0);
    }
    p.total = off;
    return p;
}

hipError_t launch_log_probs(const SoftmaxArgs& a, hipStream_t s) {
    if (a.n == 0) return hipSuccess;
    if (a.w_scales != nullptr) return log_probs<bf16_t, true>(a, s);
    return a.dtype == kDtypeBf16 ? log_probs<bf16_t, false>(a, s) : log_probs<float, false>(a, s);
}

hipError_t launch_log_probs_grad(const SoftmaxArgs& a, hipStream_t s) {
    if (a.dh == nullptr && a.dw == nullptr && a.dbias == nullptr) return hipSuccess;
    return a.dtype == kDtypeBf16 ? softmax_grad<bf16_t, true>(a, s) : softmax_grad<float, true>(a, s);
}

}  // namespace huge
