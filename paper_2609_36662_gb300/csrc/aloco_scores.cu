// Token scores: log-probabilities of given tokens, the rows' entropy and best
// alternatives, and the gradient of a loss over them.
#include <cuda_bf16.h>

#include "aloco_scores.h"
#include "aloco_tc.cuh"

namespace aloco {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kBatch = 4;            // units of a thread in flight
constexpr int kMaxSplit = 8;         // CTAs of a row
constexpr int kMostFound = 512;      // values collected for the best ones
constexpr float kLn2 = 0.693147180559945f;
// The reference of the powers of two: a whole number, so that factors between
// references are powers of two and no rounding is common to a row's terms.
constexpr float kFar = 1048576.f;    // 2^20
constexpr float kGone = -200.f;      // 2^-200 is 0 in fp32

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
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
            return __ldcs(reinterpret_cast<const uint4 *>(unit0) + u);
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
    float ref, z, s;
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

struct Found {
    unsigned long long value[kMostFound];
    int n;
    int list[kThreads], listed;
    unsigned long long warp_best[kWarps];
};

// The values of the listed threads at or above `limit`, as (order, ~index).
template <bool kBf16>
__device__ __forceinline__ void collect(const Row<kBf16> &row, int u0, int u1, unsigned limit,
                                        Found &f) {
    constexpr int N = Row<kBf16>::N;
    const int lane = threadIdx.x % 32;
    for (int i = threadIdx.x / 32; i < f.listed; i += kWarps) {
        for (int u = u0 + f.list[i] + lane * kThreads; u < u1; u += 32 * kThreads) {
            float v[N];
            Row<kBf16>::values(row.load(u, u1), v);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int j = u * N - row.phase + e;
                const unsigned o = order(v[e]);
                if (o < limit || j < 0 || j >= row.vocab) continue;
                const int at = atomicAdd(&f.n, 1);
                if (at < kMostFound) f.value[at] = (unsigned long long)o << 32 | (unsigned)~j;
            }
        }
    }
}

// The k best values of units [u0, u1), of which this thread's largest has order
// `mine`.  A limit that at least k threads' largest values reach leaves few
// values above it; only threads with one there are looked at again.
template <bool kBf16>
__device__ __forceinline__ void find_best(const Row<kBf16> &row, int u0, int u1, int k,
                                          unsigned mine, unsigned largest, Found &f,
                                          unsigned long long *best) {
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    // bisection between an order that all reach and one that fewer than k do
    __shared__ unsigned low_of[kWarps];
    const unsigned low = __reduce_min_sync(~0u, mine);
    if (lane == 0) low_of[warp] = low;
    if (tid < k) best[tid] = 0;
    __syncthreads();
    unsigned lo = low_of[0], hi = largest;
    for (int i = 1; i < kWarps; ++i) lo = min(lo, low_of[i]);
    // (the largest value alone may be reached by k threads)
    if (__syncthreads_count(mine >= hi) >= k) lo = hi;
    int slack = 8;
    for (;;) {
        while (hi - lo > 1) {
            const unsigned mid = lo + (hi - lo) / 2;
            const int c = __syncthreads_count(mine >= mid);
            if (c >= k) {
                lo = mid;
                if (c <= k + slack) break;
            } else {
                hi = mid;
            }
        }
        const unsigned limit = slack ? lo : lo + 1;
        if (tid == 0) f.n = f.listed = 0;
        __syncthreads();
        if (mine >= limit) f.list[atomicAdd(&f.listed, 1)] = tid;
        __syncthreads();
        collect(row, u0, u1, limit, f);
        __syncthreads();
        if (f.n <= kMostFound || !slack) break;
        // too many: most of them are equal to the limit.  The exact one, and
        // those above it first.
        slack = 0;
        hi = largest;
        if (lo != hi && __syncthreads_count(mine >= hi) >= k) lo = hi;
        __syncthreads();
    }
    const int n = f.n;
    if (n <= kMostFound) {
        for (int i = tid; i < n; i += kThreads) {
            const unsigned long long v = f.value[i];
            int above = 0;
            for (int j = 0; j < n; ++j) above += f.value[j] > v;
            if (above < k) best[above] = v;
        }
        if (!slack && n < k && warp == 0) {  // the rest are the first of those equal to the limit
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
        __syncthreads();
        return;
    }
    // many different values in few threads: one after another
    unsigned long long below = ~0ull;
    for (int i = 0; i < k; ++i) {
        unsigned long long top = 0;
        for (int u = u0 + tid; u < u1; u += kThreads) {
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
        if (lane == 0) f.warp_best[warp] = top;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) top = f.warp_best[w] > top ? f.warp_best[w] : top;
        if (tid == 0) best[i] = top;
        below = top;
        __syncthreads();
    }
}

// A row by a CTA or a cluster of them, read once: every thread keeps its
// maximum and its sums to a whole reference.
template <bool kBf16, bool kTop>
__global__ void __launch_bounds__(kThreads)
    token_scores_kernel(const __grid_constant__ ScoresArgs a, int split) {
    constexpr int N = Row<kBf16>::N;
    __shared__ Share share;
    __shared__ Found found;
    __shared__ float warp_ref[kWarps], warp_z[kWarps], warp_s[kWarps];
    __shared__ unsigned warp_top[kWarps];
    const int64_t r = blockIdx.x / split;
    const int rank = split > 1 ? (int)(blockIdx.x % split) : 0;
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const int64_t target = load_index(a.target, a.target_bytes, r);
    if (target < 0) {
        if (rank) return;
        if (tid == 0) {
            a.logp[r] = 0.f;
            if (a.entropy) a.entropy[r] = 0.f;
            if (a.stats) a.stats[r] = make_float2(0.f, 0.f);
        }
        if (kTop && tid < a.top) {
            a.top_ids[r * a.top + tid] = -1;
            a.top_logp[r * a.top + tid] = 0.f;
        }
        return;
    }
    const Row<kBf16> row(a.x.data + row_offset(a.x, r) * (kBf16 ? 2 : 4), a.vocab);
    const int each = (row.units + split - 1) / split;
    const int u0 = min(row.units, rank * each), u1 = min(row.units, u0 + each);

    Sums sums{-kFar, 0.f, 0.f};
    float top = -INFINITY;
    const auto pass = [&](auto term) {
        for (int u = u0 + tid; u < u1; u += kBatch * kThreads) {
            uint4 q[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) q[b] = row.load(u + b * kThreads, u1);
            term(q);
        }
    };
    pass([&](const uint4 (&q)[kBatch]) {
        const float m = Row<kBf16>::largest(q), need = ceilf(m * a.scale);
        top = max_nan(top, m);
        if (need > sums.ref) sums.refer(need);
        float z = 0.f, s = 0.f;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            float v[N];
            Row<kBf16>::values(q[b], v);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float t = fmaxf(fmaf(v[i], a.scale, -sums.ref), kGone), e = ex2(t);
                z += e;
                s = fmaf(t, e, s);
            }
        }
        sums.z += z;
        sums.s += s;
    });

    // the CTA's, then the cluster's
    const unsigned mine = order(top);
    const auto combine = [&] {
        const unsigned high = __reduce_max_sync(~0u, mine);
        const int ref = __reduce_max_sync(~0u, (int)fminf(sums.ref, 2.f * kFar));
        sums.refer((float)ref);
        const float z = warp_sum(sums.z), s = warp_sum(sums.s);
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
            for (int w = 0; w < kWarps; ++w) {
                Sums x{warp_ref[w], warp_z[w], warp_s[w]};
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
    combine();
    if constexpr (kTop) {
        if (a.top) find_best(row, u0, u1, a.top, mine, share.largest, found, share.best);
    }
    unsigned high = share.largest;
    if (split > 1) {
        cluster_sync();
        for (int p = 0; p < split; ++p) high = max(high, peer(share.largest, p));
    }
    const float m = high == ~0u ? NAN : unorder(high);
    bool far = false;                // logits so large that a whole reference does not do
    if (fabsf(m * a.scale) > kFar && fabsf(m) < INFINITY) {
        far = true;
        if (split > 1) cluster_sync();  // (all have read)
        sums = {0.f, 0.f, 0.f};
        pass([&](const uint4 (&q)[kBatch]) {
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
        combine();
        if (split > 1) cluster_sync();
    }
    if (rank == 0) {
        Sums all{share.ref, share.z, share.s};
        for (int p = 1; p < split; ++p) {
            Sums x{peer(share.ref, p), peer(share.z, p), peer(share.s, p)};
            const float to = fmaxf(all.ref, x.ref);
            all.refer(to);
            x.refer(to);
            all.z += x.z;
            all.s += x.s;
        }
        const bool bad = !(fabsf(m) < INFINITY);
        const float log2z = log2f(all.z);
        const auto log_p = [&](float x) {
            const float t = far ? (x - m) * a.scale : fmaf(x, a.scale, -all.ref);
            // (the lowest values leave fp32 in powers of two alone)
            return t < -1e30f ? (x - m) * a.inv_temp : kLn2 * (t - log2z);
        };
        if (tid == 0) {
            a.logp[r] = bad || target >= a.vocab ? NAN : log_p(row.at((int)target));
            if (a.entropy) a.entropy[r] = bad ? NAN : kLn2 * (log2z - all.s / all.z);
            if (a.stats) {
                const float z = far ? all.z : all.z * exp2f(-fmaf(m, a.scale, -all.ref));
                a.stats[r] = bad ? make_float2(NAN, NAN) : make_float2(m, z);
            }
        }
        if constexpr (kTop) {
            // an entry's place among all CTAs' is the number of larger ones
            const int n = split * a.top;
            unsigned long long v = 0;
            int place = tid;
            if (tid < n) v = split == 1 ? share.best[tid] : peer(share.best[tid % a.top], tid / a.top);
            if (split > 1) {
                if (tid < n) found.value[tid] = v;
                __syncthreads();
                place = 0;
                for (int i = 0; i < n; ++i) place += found.value[i] > v;
            }
            if (v && place < a.top) {
                a.top_ids[r * a.top + place] = bad ? -1 : (int)~(unsigned)v;
                a.top_logp[r * a.top + place] = bad ? NAN : log_p(unorder((unsigned)(v >> 32)));
            }
            // (a row with NaN may have filled fewer)
            if (bad && tid < a.top) {
                a.top_ids[r * a.top + tid] = -1;
                a.top_logp[r * a.top + tid] = NAN;
            }
        }
    }
    if (split > 1) cluster_sync();   // nobody leaves while it is read
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
template <bool kBf16>
__global__ void __launch_bounds__(kThreads)
    token_scores_grad_kernel(const __grid_constant__ ScoresArgs a, int split) {
    constexpr int N = Row<kBf16>::N, kSize = kBf16 ? 2 : 4;
    const int64_t r = blockIdx.x / split;
    const int rank = blockIdx.x % split, tid = threadIdx.x;
    const int64_t target = load_index(a.target, a.target_bytes, r);
    const bool live = target >= 0;
    const Row<kBf16> row(a.x.data + row_offset(a.x, r) * kSize, a.vocab);
    char *out = a.g.data + row_offset(a.g, r) * kSize;
    const Row<kBf16> to(out, a.vocab);
    const int each = (to.units + split - 1) / split;
    const int u0 = min(to.units, rank * each), u1 = min(to.units, u0 + each);
    const int j0 = max(0, u0 * N - to.phase), j1 = min(a.vocab, u1 * N - to.phase);

    Slope f{0.f, a.scale, 0.f, 0.f};
    int special = -1;                // this thread's element, if it is the first for it
    float value = 0.f;
    if (live) {
        const float2 st = a.stats_in[r];
        const float by_logp = a.d_logp ? a.d_logp[r] : 0.f;
        float sum = by_logp;
        if (a.d_top)
            for (int i = 0; i < a.top; ++i) {
                const int id = a.ids_in[r * a.top + i];
                if (id >= 0 && id < a.vocab) sum += a.d_top[r * a.top + i];
            }
        f.m = st.x;
        float per = 0.f;             // d_entropy (H - log z)
        if (a.d_entropy) {
            const float by_h = a.d_entropy[r];
            per = by_h * fmaf(-kLn2, log2f(st.y), a.entropy_in[r]);
            f.c1 = -by_h * kLn2 * a.inv_temp / st.y;
        }
        f.c0 = target < a.vocab ? -(sum + per) * a.inv_temp / st.y : NAN;
        const int n = 1 + (a.d_top ? a.top : 0);
        if (tid < n) {
            const auto id = [&](int i) -> int {
                return i == 0 ? (int)min(target, (int64_t)a.vocab) : a.ids_in[r * a.top + i - 1];
            };
            const int j = id(tid);
            bool mine = j >= j0 && j < j1;
            float add = 0.f;
            for (int i = 0; i < n; ++i) {
                if (id(i) != j) continue;
                if (i < tid) mine = false;
                add += i == 0 ? by_logp : a.d_top[r * a.top + i - 1];
            }
            if (mine) {
                special = j;
                value = fmaf(add, a.inv_temp, f(row.at(j)));
            }
        }
    }
    __syncthreads();                 // before the gradient covers the logits
    if (row.phase == to.phase) {
        for (int u = u0 + tid; u < u1; u += kBatch * kThreads) {
            uint4 q[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
                q[b] = live ? row.load(u + b * kThreads, u1) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int w = u + b * kThreads;
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
        for (int j = j0 + tid; j < j1; j += kThreads)
            store_one<kBf16>(out + (int64_t)j * kSize, live ? f(row.at(j)) : 0.f);
    }
    if (live) {
        __syncthreads();
        if (special >= 0) store_one<kBf16>(out + (int64_t)special * kSize, value);
    }
}

template <typename K>
cudaError_t launch(K kernel, const ScoresArgs &a, int split, bool cluster, cudaStream_t stream) {
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)(a.n * split));
    c.blockDim = dim3(kThreads);
    c.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {(unsigned)split, 1, 1};
    c.attrs = at;
    c.numAttrs = cluster && split > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&c, kernel, a, split);
}

// CTAs of a row: as many as give every SM four, of at least 512 units each.
int split_of(const ScoresArgs &a, int sm_count) {
    const int units = a.vocab / (a.bf16 ? 8 : 4);
    int split = 1;
    while (split < kMaxSplit && a.n * split < 4 * (int64_t)sm_count && units / (2 * split) >= 512)
        split *= 2;
    return split;
}

}  // namespace

cudaError_t launch_token_scores(const ScoresArgs &a, int sm_count, cudaStream_t stream) {
    const int split = split_of(a, sm_count);
    if (a.bf16)
        return a.top ? launch(token_scores_kernel<true, true>, a, split, true, stream)
                     : launch(token_scores_kernel<true, false>, a, split, true, stream);
    return a.top ? launch(token_scores_kernel<false, true>, a, split, true, stream)
                 : launch(token_scores_kernel<false, false>, a, split, true, stream);
}

cudaError_t launch_token_scores_grad(const ScoresArgs &a, int sm_count, cudaStream_t stream) {
    const int split = split_of(a, sm_count);
    return a.bf16 ? launch(token_scores_grad_kernel<true>, a, split, false, stream)
                  : launch(token_scores_grad_kernel<false>, a, split, false, stream);
}

}  // namespace aloco
