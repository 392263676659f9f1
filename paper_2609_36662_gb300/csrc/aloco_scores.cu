// Token scores: log-probabilities of given tokens, the rows' entropy and best
// alternatives, and the gradient of a loss over them.
#include <cuda_bf16.h>

#include "aloco_scores.h"
#include "aloco_tc.cuh"

namespace aloco {
namespace {

// Threads of a CTA whose groups are a warp, or the CTA itself.
constexpr int cta_of(int group) { return group == 32 ? 256 : group; }
constexpr int kBatch = 4;            // units of a thread in flight
constexpr int kMaxSplit = 8;         // CTAs of a row
constexpr int kMostFound = 512;      // values collected for the best ones
static_assert(kMostFound >= kMaxSplit * ALOCO_MAX_TOP, "a cluster's best are joined there");
constexpr float kLn2 = 0.693147180559945f;
// The reference of the powers of two: a whole number, so that factors between
// references are powers of two and no rounding is common to a row's terms.
constexpr float kFar = 1048576.f;    // 2^20
constexpr float kGone = -200.f;      // 2^-200 is 0 in fp32
constexpr float kCertain = 0.0625f;  // the other terms' share beside a nearly certain token

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two at a time.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r)
        : "l"(*reinterpret_cast<unsigned long long *>(&a)),
          "l"(*reinterpret_cast<unsigned long long *>(&b)),
          "l"(*reinterpret_cast<unsigned long long *>(&c)));
    return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(r)
        : "l"(*reinterpret_cast<unsigned long long *>(&a)),
          "l"(*reinterpret_cast<unsigned long long *>(&b)));
    return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// 2^d of a whole number d <= 0.
__device__ __forceinline__ float pow2(float d) {
    return d < -126.f ? 0.f : __int_as_float((127 + (int)d) << 23);
}
// Unsigned integers in the order of the floats; NaN above all; -0 as 0.
__device__ __forceinline__ unsigned order(float x) {
    x += 0.f;
    if (x != x) return ~0u;
    const unsigned u = __float_as_uint(x);
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unorder(unsigned k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// A row as 16-byte units of the aligned window around it: element i of unit u is
// u * N - phase + i of the row.
template <bool kBf16>
struct Row {
    static constexpr int N = kBf16 ? 8 : 4;
    const char *unit0;
    int phase, vocab, units, full0, full1;  // whole units [full0, full1)

    __device__ __forceinline__ Row(const char *p, int vocab_) : vocab(vocab_) {
        phase = (int)(((uintptr_t)p & 15) / (16 / N));
        unit0 = p - phase * (16 / N);
        units = (phase + vocab + N - 1) / N;
        full0 = phase ? 1 : 0;
        full1 = (phase + vocab) / N;
    }
    __device__ __forceinline__ float at(int j) const {
        const char *p = unit0 + (int64_t)(j + phase) * (16 / N);
        if (kBf16) return __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(p));
        return *reinterpret_cast<const float *>(p);
    }
    // the raw unit; what is not of the row is -inf
    __device__ __forceinline__ uint4 load(int u, int end) const {
        if (u >= full0 && u < full1 && u < end)
            return reinterpret_cast<const uint4 *>(unit0)[u];
        uint32_t w[4];
        const uint32_t low = kBf16 ? 0xff80ff80u : 0xff800000u;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = low;
        if (u < end) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int j = u * N - phase + i;
                if (j < 0 || j >= vocab) continue;
                if (kBf16) {
                    const uint32_t b =
                        reinterpret_cast<const uint16_t *>(unit0)[(int64_t)u * N + i];
                    w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | b << 16
                                     : (w[i / 2] & 0xffff0000u) | b;
                } else {
                    w[i] = reinterpret_cast<const uint32_t *>(unit0)[(int64_t)u * N + i];
                }
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ void values(const uint4 &q, float (&v)[N]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        if constexpr (kBf16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
        }
    }
    // values below -2^96 raised to it, -inf among them, so that products with 0 are
    // 0 (a row of nothing else is a far one)
    static __device__ __forceinline__ uint4 raised(const uint4 &q) {
        uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (kBf16) {
                const uint32_t low = 0xef80ef80u;
                const __nv_bfloat162 x = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]),
                                                 *reinterpret_cast<const __nv_bfloat162 *>(&low));
                w[i] = *reinterpret_cast<const uint32_t *>(&x);
            } else {
                w[i] = __float_as_uint(fmaxf(__uint_as_float(w[i]), -0x1p96f));
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // the largest value (NaN if there is one)
    static __device__ __forceinline__ float largest(const uint4 (&q)[kBatch]) {
        if constexpr (kBf16) {
            __nv_bfloat162 m;
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const uint32_t w[4] = {q[b].x, q[b].y, q[b].z, q[b].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&w[i]);
                    m = b + i ? __hmax2_nan(m, x) : x;
                }
            }
            return max_nan(__low2float(m), __high2float(m));
        } else {
            float m = __uint_as_float(q[0].x);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                m = max_nan(m, max_nan(__uint_as_float(q[b].x), __uint_as_float(q[b].y)));
                m = max_nan(m, max_nan(__uint_as_float(q[b].z), __uint_as_float(q[b].w)));
            }
            return m;
        }
    }
};

__device__ __forceinline__ int64_t row_offset(const Rows &r, int64_t row) {
    const int64_t b = row / r.per_batch;
    return b * r.batch_stride + (row - b * r.per_batch) * r.row_stride;
}
__device__ __forceinline__ int64_t load_index(const void *p, int bytes, int64_t i) {
    return bytes == 8 ? static_cast<const int64_t *>(p)[i] : static_cast<const int32_t *>(p)[i];
}

// z = sum 2^t, s = sum t 2^t with t = x scale - ref.
struct Sums {
    float ref, z, s;
    __device__ __forceinline__ void add(float t) {
        const float e = ex2(t);
        z += e;
        s = fmaf(t, e, s);
    }
    __device__ __forceinline__ void take_away(float t) {  // (one value alone leaves 0)
        const float e = ex2(t);
        z -= e;
        s -= __fmul_rn(t, e);
    }
    __device__ __forceinline__ void refer(float to) {   // to >= ref, both whole
        const float d = ref - to, f = pow2(d);
        s = f == 0.f ? 0.f : fmaf(d, z, s) * f;
        z *= f;
        ref = to;
    }
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

// One CTA's share of a row, as the others of its cluster read it.
struct Share {
    unsigned largest;
    float ref, z, s;                 // without the largest's term, where rows are split
    int owner;                       // the thread that read the row's largest value
    unsigned long long best[ALOCO_MAX_TOP];  // (order, ~index), largest first; 0: none
};

template <typename T>
__device__ __forceinline__ T peer(const T &mine, int rank) {
    const uint32_t at = cluster_addr(smem_addr(&mine), rank);
    if constexpr (sizeof(T) == 8) {
        unsigned long long v;
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
        return v;
    } else {
        uint32_t v;
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
        T r;
        memcpy(&r, &v, 4);
        return r;
    }
}

// A group of threads that takes a row together: a CTA, or a warp of it.
template <int kGroup>
struct Group {
    static constexpr int kWarps = kGroup / 32;
    static __device__ __forceinline__ int thread() { return threadIdx.x % kGroup; }
    static __device__ __forceinline__ int index() { return threadIdx.x / kGroup; }
    static __device__ __forceinline__ void sync() {
        if constexpr (kGroup == 32)
            __syncwarp();
        else
            __syncthreads();
    }
    static __device__ __forceinline__ int count(bool is) {
        if constexpr (kGroup == 32)
            return __popc(__ballot_sync(~0u, is));
        else
            return __syncthreads_count(is);
    }
};

template <int kGroup>
struct Found {
    static constexpr int kList = 2 * kGroup;
    unsigned long long value[kMostFound];
    int n;
    int list[kList], listed;
    unsigned low[Group<kGroup>::kWarps];
    unsigned long long best[Group<kGroup>::kWarps];

    __device__ __forceinline__ void add(unsigned o, int j) {
        const int at = atomicAdd(&n, 1);
        if (at < kMostFound) value[at] = (unsigned long long)o << 32 | (unsigned)~j;
    }
};

// The largest of a thread's batches, where two of them were, and the third.
struct Largest {
    float first = -INFINITY, second = -INFINITY, third = -INFINITY;
    int at_first = 0, at_second = 0;
    __device__ __forceinline__ void take(float m, int turn) {
        if (m > first) {
            third = second;
            second = first;
            at_second = at_first;
            first = m;
            at_first = turn;
        } else if (m > second) {
            third = second;
            second = m;
            at_second = turn;
        } else {
            third = fmaxf(third, m);
        }
    }
};

// A lower limit that at least k of the row's values reach: the c-th largest of
// the lanes' batches (up to three of a lane) in every warp that is full, the least
// of these.  `mine`: the order of this thread's maximum.
template <int kGroup>
__device__ __forceinline__ unsigned lower_limit(unsigned mine, const Largest &large, int units,
                                                int k, Found<kGroup> &f) {
    using G = Group<kGroup>;
    const int full = min(units / 32, G::kWarps), lane = threadIdx.x % 32;
    unsigned x = mine, x2 = order(large.second), x3 = order(large.third), c = 0;
    if (full > 0)
        for (int i = (k + full - 1) / full; i > 0; --i) {
            c = __reduce_max_sync(~0u, x);
            if (lane == __ffs(__ballot_sync(~0u, x == c)) - 1) x = x2, x2 = x3, x3 = 0;
        }
    if constexpr (kGroup == 32) return c;
    if (lane == 0) f.low[G::thread() / 32] = c;
    __syncthreads();
    unsigned low = full > 0 ? f.low[0] : 0;
    for (int i = 1; i < full; ++i) low = min(low, f.low[i]);
    return low;
}

// The values of a unit at or above `limit`, as (order, ~index).
template <bool kBf16, int kGroup>
__device__ __forceinline__ void collect(const Row<kBf16> &row, int u, int u1, unsigned limit,
                                        Found<kGroup> &f) {
    constexpr int N = Row<kBf16>::N;
    float v[N];
    Row<kBf16>::values(row.load(u, u1), v);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const int j = u * N - row.phase + e;
        const unsigned o = order(v[e]);
        if (o >= limit && u < u1 && j >= 0 && j < row.vocab) f.add(o, j);
    }
}

// Every collected value's place is the number of larger ones.
template <int kGroup>
__device__ __forceinline__ void place(const Found<kGroup> &f, int n, int k,
                                      unsigned long long *best) {
    for (int i = Group<kGroup>::thread(); i < n; i += kGroup) {
        const unsigned long long v = f.value[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += f.value[j] > v;
        if (above < k) best[above] = v;
    }
}

// The k best values of units [u0, u1) where a first limit leaves too many (equal
// values throughout; everything worth having in few places): of the threads' maxima
// (`mine`) an exact limit that k of them reach is found by bisection, and threads above
// it are read again.
template <bool kBf16, int kGroup>
__device__ __noinline__ void find_best(const Row<kBf16> &row, int u0, int u1, int k, unsigned mine,
                                       unsigned largest, Found<kGroup> &f,
                                       unsigned long long *best) {
    using G = Group<kGroup>;
    const int tid = G::thread(), lane = tid % 32, warp = tid / 32;
    const unsigned low = __reduce_min_sync(~0u, mine);
    if (lane == 0) f.low[warp] = low;
    G::sync();
    unsigned lo = f.low[0], hi = largest;
    for (int i = 1; i < G::kWarps; ++i) lo = min(lo, f.low[i]);
    // lo: an order that k threads reach, hi: one that fewer do
    if (G::count(mine >= hi) >= k) lo = hi;
    while (hi - lo > 1) {
        const unsigned mid = lo + (hi - lo) / 2;
        if (G::count(mine >= mid) >= k)
            lo = mid;
        else
            hi = mid;
    }
    for (int above = 0; above < 2; ++above) {   // all that reach it; those above it
        G::sync();
        if (tid == 0) f.n = f.listed = 0;
        G::sync();
        if (mine >= lo + above) f.list[atomicAdd(&f.listed, 1)] = tid;
        G::sync();
        for (int i = warp; i < f.listed; i += G::kWarps)
            for (int u = u0 + f.list[i] + lane * kGroup; u < u1; u += 32 * kGroup)
                collect<kBf16, kGroup>(row, u, u1, lo + above, f);
        G::sync();
        const int n = f.n;
        if (n > kMostFound) continue;
        place(f, n, k, best);
        if (above && n < k && warp == 0) {  // the rest are the first of those equal to it
            int have = n;
            const int from = max(0, u0 * Row<kBf16>::N - row.phase);
            const int to = min(row.vocab, u1 * Row<kBf16>::N - row.phase);
            for (int j = from; j < to && have < k; j += 32) {
                const bool is = j + lane < to && order(row.at(j + lane)) == lo;
                const unsigned which = __ballot_sync(~0u, is);
                const int at = have + __popc(which & ((1u << lane) - 1));
                if (is && at < k) best[at] = (unsigned long long)lo << 32 | (unsigned)~(j + lane);
                have += __popc(which);
            }
        }
        G::sync();
        return;
    }
    // many different values in few threads: one after another
    unsigned long long below = ~0ull;
    for (int i = 0; i < k; ++i) {
        unsigned long long top = 0;
        for (int u = u0 + tid; u < u1; u += kGroup) {
            float v[Row<kBf16>::N];
            Row<kBf16>::values(row.load(u, u1), v);
#pragma unroll
            for (int e = 0; e < Row<kBf16>::N; ++e) {
                const int j = u * Row<kBf16>::N - row.phase + e;
                const unsigned long long p =
                    (unsigned long long)order(v[e]) << 32 | (unsigned)~j;
                if (j >= 0 && j < row.vocab && p < below && p > top) top = p;
            }
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const unsigned long long o = __shfl_xor_sync(~0u, top, d);
            top = o > top ? o : top;
        }
        if (lane == 0) f.best[warp] = top;
        G::sync();
        for (int w = 0; w < G::kWarps; ++w) top = f.best[w] > top ? f.best[w] : top;
        if (tid == 0) best[i] = top;
        below = top;
        G::sync();
    }
}

// A row by a warp, a CTA or a cluster of them, read once: every thread keeps its
// maxima and its sums to a whole reference.  For the alternatives the maxima give
// a limit that k values reach, and the few batches that reach it are read again.
//
// kSplit: rows of more than one CTA.  (Where there are none `split` stays a value that the
// compiler does not know: one that it knows makes the loop's values spill, in fp32 still
// and at first in bf16 too, 84 us in place of 80.)
//
// Bound by HBM; the steps behind a row's last unit (a limit, a few values read
// again, their order: about 2 us) are hidden by the other CTAs of the SM, so CTAs
// are small.  8184 x 32000 bf16 with 8 alternatives: 104 us with 11 CTAs of 128
// threads an SM, 120 with 6 of 256 (77 at the copy rate); 4000 x 128256: 179 and
// 182 us (152), 170 with 9 CTAs, which take 72 us where 11 take 59 for 1533 x 50257
// fp32.  Without alternatives 10 are best: 88 and 159 us.
template <bool kBf16, bool kTop, int kGroup, bool kSplit>
__global__ void __launch_bounds__(cta_of(kGroup), kGroup == 32 ? 4 : kSplit ? 8 : kTop ? 11 : 10)
    token_scores_kernel(const __grid_constant__ ScoresArgs a, int split) {
    using G = Group<kGroup>;
    constexpr int N = Row<kBf16>::N, kGroups = cta_of(kGroup) / kGroup, kWarps = G::kWarps;
    __shared__ Share shares[kGroups];
    __shared__ Found<kGroup> founds[kTop ? kGroups : 1];
    __shared__ float warp_refs[kGroups][kWarps], warp_zs[kGroups][kWarps], warp_ss[kGroups][kWarps];
    __shared__ unsigned warp_tops[kGroups][kWarps];
    const int group = G::index();
    Share &share = shares[group];
    Found<kGroup> &found = founds[kTop ? group : 0];
    const int r = kGroup == 32 ? (int)blockIdx.x * kGroups + group : (int)blockIdx.x / split;
    const int rank = split > 1 ? (int)(blockIdx.x % split) : 0;
    const int tid = G::thread(), lane = tid % 32, warp = tid / 32;
    if (r >= a.n) return;
    // (in 32 bits, as r is: with either in 64 the loop's values spill)
    const int target = (int)max((int64_t)-1, min(load_index(a.target, a.target_bytes, r),
                                                 (int64_t)a.vocab));
    if (target < 0) {
        if (rank) return;
        if (tid == 0) {
            a.logp[r] = 0.f;
            if (a.entropy) a.entropy[r] = 0.f;
            if (a.stats) a.stats[r] = make_float2(0.f, 0.f);
        }
        if (kTop && tid < a.top) {
            a.top_ids[(int64_t)r * a.top + tid] = -1;
            a.top_logp[(int64_t)r * a.top + tid] = 0.f;
        }
        return;
    }
    const Row<kBf16> row(a.x.data + row_offset(a.x, r) * (kBf16 ? 2 : 4), a.vocab);
    const int each = (row.units + split - 1) / split;
    const int u0 = min(row.units, rank * each), u1 = min(row.units, u0 + each);

    Sums sums{-kFar, 0.f, 0.f};
    Largest large;
    bool nan = false;
    const auto pass = [&](auto term) {
        int turn = 0;
        for (int u = u0 + tid; u - tid < u1; u += kBatch * kGroup, ++turn) {
            uint4 q[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) q[b] = row.load(u + b * kGroup, u1);
            term(q, u, turn);
        }
    };
    pass([&](const uint4 (&q)[kBatch], int, int turn) {
        const float m = Row<kBf16>::largest(q), need = ceilf(m * a.scale);
        nan |= m != m;
        large.take(m, turn);
        if (need > sums.ref) sums.refer(need);
        float2 z = {0.f, 0.f}, s = {0.f, 0.f};
        const float2 scale = {a.scale, a.scale}, ref = {-sums.ref, -sums.ref};
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            float v[N];
            Row<kBf16>::values(Row<kBf16>::raised(q[b]), v);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                // (2^t is 0 where x was raised: t is below -2^60 there)
                const float2 t = fma2({v[i], v[i + 1]}, scale, ref), e = {ex2(t.x), ex2(t.y)};
                z = add2(z, e);
                s = fma2(t, e, s);
            }
        }
        sums.z += z.x + z.y;
        sums.s += s.x + s.y;
    });

    // A value's power (of -inf one whose term is 0).  Logits so large that a whole
    // reference does not do, far ones, have the largest as theirs.
    bool far = false;
    float m = 0.f;
    const auto power = [&](float x, float ref) {
        return far ? fmaxf((x - m) * a.scale, kGone) : fmaf(fmaxf(x, -0x1p96f), a.scale, -ref);
    };
    // The log-probability of a token that is nearly certain is what the other terms are to
    // it, which a sum with its term has rounded away: where they are a sixteenth at most
    // the units of the thread that had it are taken again without it.
    const auto certain = [](float z, float e) { return z - e < kCertain * z; };
    const auto take_again = [&](int u, int step, float without, float ref) {
        for (; u < u1; u += step) {
            float v[N];
            Row<kBf16>::values(row.load(u, u1), v);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float t = power(v[i], ref), e = v[i] == without ? 0.f : ex2(t);
                sums.z += e;
                sums.s = fmaf(t, e, sums.s);
            }
        }
    };
    // The group's sums.  Where rows are split every warp sees to its own largest value,
    // which costs no barrier more; else the row's is seen to below (by warps: 189 us in
    // place of 184 for 4000 x 128256 bf16, 60 in place of 55 for 1533 x 50257 fp32; by the
    // row where it is split: 300 x 50257 bf16, all nearly certain, 26 us in place of 20).
    const unsigned mine = nan ? ~0u : order(large.first);
    const auto combine = [&] {
        const unsigned high = __reduce_max_sync(~0u, mine);
        const int ref = __reduce_max_sync(~0u, (int)fminf(sums.ref, 2.f * kFar));
        sums.refer((float)ref);
        Sums all{(float)ref, warp_sum(sums.z), warp_sum(sums.s)};
        if constexpr (kSplit) {
            const float top = unorder(high), t = power(top, all.ref);
            if (certain(all.z, ex2(t))) {
                const int owner = __ffs(__ballot_sync(~0u, mine == high)) - 1;
                if (lane == owner) sums.z = sums.s = 0.f;
                take_again(u0 + tid - lane + owner + lane * kGroup, 32 * kGroup, top, all.ref);
                all = {all.ref, warp_sum(sums.z), warp_sum(sums.s)};
            } else {
                all.take_away(t);
            }
        }
        const float z = all.z, s = all.s;
        if constexpr (kGroup == 32) {
            if (lane == 0) {
                share.largest = high;
                share.ref = (float)ref;
                share.z = z;
                share.s = s;
            }
            __syncwarp();
            return;
        }
        float *warp_ref = warp_refs[group], *warp_z = warp_zs[group], *warp_s = warp_ss[group];
        unsigned *warp_top = warp_tops[group];
        if (lane == 0) {
            warp_top[warp] = high;
            warp_ref[warp] = (float)ref;
            warp_z[warp] = z;
            warp_s[warp] = s;
        }
        __syncthreads();
        if (tid == 0) {
            unsigned h = 0;
            float to = -kFar;
            for (int w = 0; w < kWarps; ++w) {
                h = max(h, warp_top[w]);
                to = fmaxf(to, warp_ref[w]);
            }
            Sums all{to, 0.f, 0.f};
            bool missing = kSplit;   // the largest has not come yet
            for (int w = 0; w < kWarps; ++w) {
                Sums x{warp_ref[w], warp_z[w], warp_s[w]};
                if (missing && warp_top[w] == h)
                    missing = false;
                else if (kSplit)
                    x.add(power(unorder(warp_top[w]), x.ref));
                x.refer(to);
                all.z += x.z;
                all.s += x.s;
            }
            share.largest = h;
            share.ref = all.ref;
            share.z = all.z;
            share.s = all.s;
        }
        __syncthreads();
    };
    if constexpr (kTop) {
        if (tid < a.top) share.best[tid] = 0;
        if (tid == 0) found.n = found.listed = 0;
    }
    combine();
    if constexpr (kTop) {
        const unsigned limit = lower_limit<kGroup>(mine, large, u1 - u0, a.top, found);
        constexpr int kList = Found<kGroup>::kList;
        if (mine >= limit) {
            const int turns = (u1 - u0 + kBatch * kGroup - 1) / (kBatch * kGroup);
            const bool all = order(large.third) >= limit && turns > 2;
            const int n = all ? turns : turns > 1 && order(large.second) >= limit ? 2 : 1;
            const int at = atomicAdd(&found.listed, n);
            for (int i = 0; i < n && at + i < kList; ++i)
                found.list[at + i] =
                    tid | (all ? i : i ? large.at_second : large.at_first) << 16;
        }
        G::sync();
        const int listed = found.listed;
        if (listed <= kList)
            for (int i = tid; i < listed * kBatch; i += kGroup) {
                const int entry = found.list[i / kBatch];
                collect<kBf16, kGroup>(row, u0 + (entry & 0xffff) +
                                                ((entry >> 16) * kBatch + i % kBatch) * kGroup,
                                       u1, limit, found);
            }
        G::sync();
        const int n = found.n;
        if (listed > kList || n > kMostFound)
            find_best<kBf16, kGroup>(row, u0, u1, a.top, mine, share.largest, found, share.best);
        else
            place(found, n, a.top, share.best);
        G::sync();
    }
    unsigned high = share.largest;
    if constexpr (kSplit) {
        cluster_sync();
        high = __reduce_max_sync(~0u, lane < split ? peer(share.largest, lane) : 0);
    }
    m = high == ~0u ? NAN : unorder(high);
    const bool bad = !(fabsf(m) < INFINITY);
    far = !bad && fabsf(m * a.scale) > kFar;
    if (far) {
        sums = {0.f, 0.f, 0.f};
        pass([&](const uint4 (&q)[kBatch], int, int) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                float v[N];
                Row<kBf16>::values(q[b], v);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float t = fmaxf((v[i] - m) * a.scale, kGone), e = ex2(t);
                    sums.z += e;
                    sums.s = fmaf(t, e, sums.s);
                }
            }
        });
        if constexpr (kSplit) cluster_sync();  // (all have read)
        combine();
        if constexpr (kSplit) cluster_sync();
    }
    // The other terms' sums.
    Sums others{-kFar, 0.f, 0.f};
    if constexpr (kSplit) {          // a lane reads a CTA's
        const unsigned top = lane < split ? peer(share.largest, lane) : 0;
        const int first = __ffs(__ballot_sync(~0u, top == high)) - 1;
        if (lane < split) {
            others = {peer(share.ref, lane), peer(share.z, lane), peer(share.s, lane)};
            if (lane != first) others.add(power(unorder(top), others.ref));
        }
        others.refer((float)__reduce_max_sync(~0u, (int)others.ref));
        others.z = warp_sum(others.z);
        others.s = warp_sum(others.s);
    } else {
        others = {share.ref, share.z, share.s};
    }
    const float t_m = power(m, others.ref), e_m = ex2(t_m);
    if constexpr (!kSplit) {
        // (8 x 1023 x 32000 bf16, of which 12 % are nearly certain: 80.0 us, 78.1 with the
        // sum of all; 81.1 where the limit is an eighth)
        if (!bad && certain(others.z, e_m)) {
            sums.refer(others.ref);
            if (mine == high) {
                share.owner = tid;
                sums.z = sums.s = 0.f;
            }
            G::sync();
            take_again(u0 + share.owner + tid * kGroup, kGroup * kGroup, m, others.ref);
            __syncwarp();
            combine();
            others = {share.ref, share.z, share.s};
        } else {
            others.take_away(t_m);
        }
        if (warp) return;            // the first warp does the rest
    }
    if (rank == 0) {
        if constexpr (kTop && kSplit) {
            for (int i = tid; i < split * a.top; i += kGroup)
                found.value[i] = peer(share.best[i % a.top], i / a.top);
            __syncthreads();
        }
        // The log-probability of the largest is -log(1 + r), r the other terms to it, and the
        // entropy log(1 + r) and what the others' powers lie below its own: of parts that
        // are not below 0, so that neither has the wrong sign where one token has all.
        // (sum (t_j - t_m) 2^t_j over the others, which is not above 0)
        const float below = fminf(fmaf(-t_m, others.z, others.s), 0.f);
        // One float for log2(e) / tau puts the same relative error on all powers of a call,
        // which sums over many rows' logp would keep: sum 2^(t (1 + d)) is sum 2^t + d ln 2
        // sum t 2^t to first order (d < 2^-24, t < 126).  (What ex2 loses on average,
        // 5e-8, is in both of z and e_m.)
        const float to_m = fmaf(a.tilt, below, others.z) / e_m, log_z = log1pf(to_m);
        const auto log_p = [&](float x) { return fmaf(x - m, a.inv_temp, -log_z); };
        if (tid == 0) {
            a.logp[r] = bad || target >= a.vocab ? NAN : log_p(row.at(target));
            if (a.entropy)
                a.entropy[r] = bad ? NAN : fmaf(-kLn2, below / (others.z + e_m), log_z);
            if (a.stats) a.stats[r] = bad ? make_float2(NAN, NAN) : make_float2(m, 1.f + to_m);
        }
        if constexpr (kTop) {
            const int n = bad ? a.top : split * a.top;
            for (int i = tid; i < n; i += kGroup) {
                // an entry's place among all CTAs' is the number of larger ones (a row with
                // NaN may have fewer)
                unsigned long long v = 0;
                int place = i;
                if (!bad) {
                    v = kSplit ? found.value[i] : share.best[i];
                    if constexpr (kSplit) {
                        place = 0;
                        for (int o = 0; o < n; ++o) place += found.value[o] > v;
                    }
                    if (!v || place >= a.top) continue;
                }
                a.top_ids[(int64_t)r * a.top + place] = bad ? -1 : (int)~(unsigned)v;
                a.top_logp[(int64_t)r * a.top + place] = bad ? NAN : log_p(unorder((unsigned)(v >> 32)));
            }
        }
    }
    if constexpr (kSplit) cluster_sync();  // nobody leaves while it is read
}

// ------------------------------------------------------------------ gradient

// p (c0 + c1 t) with p = 2^t / z and t = (x - largest) scale.
struct Slope {
    float m, scale, c0, c1;
    __device__ __forceinline__ float operator()(float x) const {
        const float t = fmaxf((x - m) * scale, kGone);
        return ex2(t) * fmaf(c1, t, c0);
    }
};

template <bool kBf16>
__device__ __forceinline__ void store_one(char *p, float v) {
    if (kBf16)
        *reinterpret_cast<__nv_bfloat16 *>(p) = __float2bfloat16_rn(v);
    else
        *reinterpret_cast<float *>(p) = v;
}

// A row's units, read and written once; the token's and the alternatives'
// elements are worked out before and written last.
template <bool kBf16, int kGroup>
__global__ void __launch_bounds__(cta_of(kGroup))
    token_scores_grad_kernel(const __grid_constant__ ScoresArgs a, int split) {
    using G = Group<kGroup>;
    constexpr int N = Row<kBf16>::N, kSize = kBf16 ? 2 : 4;
    const int64_t r = kGroup == 32 ? (int64_t)blockIdx.x * (cta_of(kGroup) / kGroup) + G::index()
                                   : blockIdx.x / split;
    const int rank = split > 1 ? (int)(blockIdx.x % split) : 0, tid = G::thread();
    if (r >= a.n) return;
    const int64_t target = load_index(a.target, a.target_bytes, r);
    const bool live = target >= 0;
    const Row<kBf16> row(a.x.data + row_offset(a.x, r) * kSize, a.vocab);
    char *out = a.g.data + row_offset(a.g, r) * kSize;
    const Row<kBf16> to(out, a.vocab);
    const int each = (to.units + split - 1) / split;
    const int u0 = min(to.units, rank * each), u1 = min(to.units, u0 + each);
    const int j0 = max(0, u0 * N - to.phase), j1 = min(a.vocab, u1 * N - to.phase);
    const bool same = row.phase == to.phase;

    uint4 q[kBatch];                 // the first units come while the factors do
    const auto load = [&](int u) {
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
            q[b] = live ? row.load(u + b * kGroup, u1) : make_uint4(0, 0, 0, 0);
    };
    if (same) load(u0 + tid);

    Slope f{0.f, a.scale, 0.f, 0.f};
    int special = -1, spare = -1;    // this thread's elements, if it is the first for them
    float value = 0.f, spare_value = 0.f;
    if (live) {
        const float2 st = a.stats_in[r];
        const int n = 1 + (a.d_top ? a.top : 0);
        // lane i has the i-th element's index and gradient (lane 0 the 32nd
        // alternative's too)
        const int lane = threadIdx.x % 32;
        int id = -1, id32 = -1;
        float by = 0.f, by32 = 0.f;
        if (lane == 0) {
            id = (int)min(target, (int64_t)a.vocab);
            by = a.d_logp ? a.d_logp[r] : 0.f;
            if (n == 33) {
                id32 = a.ids_in[r * 32 + 31];
                by32 = a.d_top[r * 32 + 31];
            }
        } else if (lane < n) {
            id = a.ids_in[r * a.top + lane - 1];
            by = a.d_top[r * a.top + lane - 1];
        }
        id32 = __shfl_sync(~0u, id32, 0);
        by32 = __shfl_sync(~0u, by32, 0);
        // sums in the order of the elements: of all, and of those with this
        // thread's index
        const int j = tid == 32 ? id32 : id;
        bool mine = tid < n && j >= j0 && j < j1;
        float sum = 0.f, add = 0.f;
        for (int i = 0; i < n; ++i) {
            const int jj = i < 32 ? __shfl_sync(~0u, id, i) : id32;
            const float g = i < 32 ? __shfl_sync(~0u, by, i) : by32;
            if (i == 0 || (jj >= 0 && jj < a.vocab)) sum += g;
            if (jj != j) continue;
            if (i < tid) mine = false;
            add += g;
        }
        f.m = st.x;
        float per = 0.f;             // d_entropy (H - log z)
        if (a.d_entropy) {
            const float by_h = a.d_entropy[r];
            per = by_h * fmaf(-kLn2, log2f(st.y), a.entropy_in[r]);
            f.c1 = -by_h * kLn2 * a.inv_temp / st.y;
        }
        f.c0 = target < a.vocab ? -(sum + per) * a.inv_temp / st.y : NAN;
        if (mine) {
            special = j;
            value = fmaf(add, a.inv_temp, f(row.at(j)));
        }
        // (a warp's 33rd element has no lane of its own)
        if (kGroup == 32 && n == 33 && lane == 0) {
            bool first = id32 >= j0 && id32 < j1;
            for (int i = 0; i < 32; ++i) {
                const int jj = i ? a.ids_in[r * 32 + i - 1] : id;
                if (jj == id32) first = false;
            }
            if (first) {
                spare = id32;
                spare_value = fmaf(by32, a.inv_temp, f(row.at(id32)));
            }
        }
    }
    G::sync();                       // before the gradient covers the logits
    if (same) {
        for (int u = u0 + tid; u < u1; u += kBatch * kGroup) {
            if (u != u0 + tid) load(u);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int w = u + b * kGroup;
                if (w >= u1) break;
                float v[N];
                Row<kBf16>::values(q[b], v);
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = live ? f(v[i]) : 0.f;
                if (w >= to.full0 && w < to.full1) {
                    uint4 o;
                    if constexpr (kBf16) {
                        uint32_t *p = &o.x;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                            p[i] = *reinterpret_cast<const uint32_t *>(&h);
                        }
                    } else {
                        o = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]),
                                       __float_as_uint(v[2]), __float_as_uint(v[3]));
                    }
                    __stcs(reinterpret_cast<uint4 *>(const_cast<char *>(to.unit0)) + w, o);
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int j = w * N - to.phase + i;
                        if (j >= 0 && j < a.vocab) store_one<kBf16>(out + (int64_t)j * kSize, v[i]);
                    }
                }
            }
        }
    } else {
        for (int j = j0 + tid; j < j1; j += kGroup)
            store_one<kBf16>(out + (int64_t)j * kSize, live ? f(row.at(j)) : 0.f);
    }
    if (live) {
        G::sync();
        if (special >= 0) store_one<kBf16>(out + (int64_t)special * kSize, value);
        if (spare >= 0) store_one<kBf16>(out + (int64_t)spare * kSize, spare_value);
    }
}

template <typename K>
cudaError_t launch(K kernel, const ScoresArgs &a, int group, int split, bool cluster,
                   cudaStream_t stream) {
    cudaLaunchConfig_t c{};
    const int rows = cta_of(group) / group;
    c.gridDim = dim3((unsigned)((a.n + rows - 1) / rows * split));
    c.blockDim = dim3(cta_of(group));
    c.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {(unsigned)split, 1, 1};
    c.attrs = at;
    c.numAttrs = cluster && split > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&c, kernel, a, split);
}

// Who takes a row: a warp, a CTA, or `split` CTAs.
struct Shape {
    int group, split;
};
Shape shape_of(const ScoresArgs &a, int sm_count, int cta, int ctas_per_sm) {
    const int units = a.vocab / (a.bf16 ? 8 : 4);
    // 20000 x 4096 bf16 with 8 alternatives: 52 us by warps, 178 by CTAs; 4000 x 8192:
    // 26 and 39 us.  Few rows do not fill the SMs with warps.
    if (units <= 1024 && (units <= 128 || a.n >= 8 * (int64_t)sm_count)) return {32, 1};
    int split = 1;
    while (split < kMaxSplit && a.n * split < ctas_per_sm * (int64_t)sm_count &&
           units / (2 * split) >= 512)
        split *= 2;
    return {cta, split};
}

template <bool kBf16, bool kTop>
cudaError_t launch_scores(const ScoresArgs &a, const Shape &s, cudaStream_t stream) {
    if (s.group == 32)
        return launch(token_scores_kernel<kBf16, kTop, 32, false>, a, 32, 1, false, stream);
    return s.split > 1
               ? launch(token_scores_kernel<kBf16, kTop, 128, true>, a, 128, s.split, true, stream)
               : launch(token_scores_kernel<kBf16, kTop, 128, false>, a, 128, 1, true, stream);
}
template <bool kBf16>
cudaError_t launch_grad(const ScoresArgs &a, const Shape &s, cudaStream_t stream) {
    return s.group == 32 ? launch(token_scores_grad_kernel<kBf16, 32>, a, 32, 1, false, stream)
                         : launch(token_scores_grad_kernel<kBf16, 256>, a, 256, s.split, false,
                                  stream);
}

}  // namespace

cudaError_t launch_token_scores(const ScoresArgs &a, int sm_count, cudaStream_t stream) {
    // (clusters wait for one another: only where rows are few)
    const Shape s = shape_of(a, sm_count, 128, 8);
    if (a.bf16)
        return a.top ? launch_scores<true, true>(a, s, stream)
                     : launch_scores<true, false>(a, s, stream);
    return a.top ? launch_scores<false, true>(a, s, stream)
                 : launch_scores<false, false>(a, s, stream);
}

cudaError_t launch_token_scores_grad(const ScoresArgs &a, int sm_count, cudaStream_t stream) {
    // parts of a row are their own here, and short CTAs end together: 1533 x 50257
    // fp32 107 us with 4 an SM, 100 with 32; 111 with 64
    const Shape s = shape_of(a, sm_count, 256, 32);
    return a.bf16 ? launch_grad<true>(a, s, stream) : launch_grad<false>(a, s, stream);
}

}  // namespace aloco
