// Log-probabilities of tokens, and the policy and preference losses with their
// gradients by the logits.
//
// A row x[0..V) with its token a and temperature tau:
//   m = max x,  z = sum_j exp((x_j - m) / tau),
//   logp = (x_a - m) / tau - log z,   p_j = exp((x_j - m) / tau) / z
//   dL/dx_j = k ([j = a] - p_j),  k = dL/dlogp / tau.
//
// Row kernel: persistent clusters take the rows in turn.  Each CTA has a
// producer warp that copies its part of the rows ahead into a ring in shared
// memory (cp.async.bulk), so that HBM is read while the consumers compute,
// reduce and store; the consumers take a row's part into registers, turn it
// into exp((x - own maximum) / tau) once, and reduce (maximum, sum) pairs over
// warp, CTA and, through distributed shared memory, the cluster.  The gradient
// is each kept value times one factor per thread: the logits are read once and
// the gradient is written once.
// The preference loss needs every row of a pair before any of its gradients:
// its first kernel leaves m and 1/z of every row, its second (in small calls
// the first one's last cluster) adds the log ratios, and its third reads the logits
// again.
//
// What bounds them is HBM, and for vocabularies of more than one CTA the
// exchange within the cluster.  Whole calls, of the copy rate: policy 8 x 1023 x
// 32000 bf16 without prompt rows 164 us, 0.94; 8 x 1000 x 128256 644 us, 0.89;
// log-probabilities 4 x 1023 x 128256 131 us, 0.89; preference 16 sequences to
// 1024 x 32000 335 us, 0.86 of its bytes with the logits read twice.
//
// A row may start off a 16-byte boundary (odd vocabularies): the units are
// those of the aligned window around it; whole ones are copied, and the two at
// its ends are read and written element by element.
#pragma once

#include <limits.h>

#include <cooperative_groups.h>

#include "aloco_bulk.cuh"
#include "aloco_logits.h"
#include "aloco_marks.cuh"
#include "aloco_sync_kernel.cuh"
#include "aloco_units.cuh"

namespace aloco {

namespace {

namespace cg = cooperative_groups;

// Wait until the kernel before this one in the stream has completed (at once
// where this launch is not serialised programmatically).
__device__ __forceinline__ void wait_for_previous() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// What a row kernel leaves: log-probabilities, also a gradient, the same where
// the gradient's rows may lie otherwise to the 16-byte boundaries than the
// logits' do, what the preference loss needs of a row, or its gradient.
// (kPolicySmall: see finishes.)
constexpr int kFwd = 0, kPolicy = 1, kPolicyShifted = 2, kPref = 3, kGrad = 4, kGradShifted = 5,
              kPolicySmall = 6;
constexpr bool is_policy(int mode) {
    return mode == kPolicy || mode == kPolicyShifted || mode == kPolicySmall;
}
constexpr bool is_grad(int mode) { return mode == kGrad || mode == kGradShifted; }
constexpr bool writes_grad(int mode) { return is_policy(mode) || is_grad(mode); }
constexpr bool may_shift(int mode) { return mode == kPolicyShifted || mode == kGradShifted; }

template <bool BF16>
struct Unit {
    static constexpr int kSize = BF16 ? 2 : 4;    // bytes of an element
    static constexpr int kElems = 16 / kSize;     // elements of a unit
};

// Elements of a row by 16-byte units of the window around it.
struct Window {
    char *base;   // 16-byte aligned
    int head;     // elements of the window before the row
    int end;      // head + vocab
    int units;
};

template <bool BF16>
__device__ __forceinline__ Window window_at(char *base, int head, int vocab) {
    const int end = head + vocab;
    return {base, head, end, (end + Unit<BF16>::kElems - 1) / Unit<BF16>::kElems};
}
template <bool BF16>
__device__ __forceinline__ Window window_of(const Rows &r, int64_t row, int vocab) {
    const uint32_t per = (uint32_t)r.per_batch, b = (uint32_t)row / per;  // rows < 2^31
    char *p = r.data + ((int64_t)b * r.batch_stride +
                        (int64_t)((uint32_t)row - b * per) * r.row_stride) * Unit<BF16>::kSize;
    const int off = (int)((uintptr_t)p & 15);
    return window_at<BF16>(p - off, off / Unit<BF16>::kSize, vocab);
}

template <bool BF16>
__device__ __forceinline__ float load1(const char *base, int e) {
    if constexpr (BF16)
        return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(base)[e] << 16);
    else
        return reinterpret_cast<const float *>(base)[e];
}
template <bool BF16>
__device__ __forceinline__ void store1(char *base, int e, float v) {
    if constexpr (BF16)
        reinterpret_cast<__nv_bfloat16 *>(base)[e] = __float2bfloat16_rn(v);
    else
        reinterpret_cast<float *>(base)[e] = v;
}

// One 16-byte unit of a row's elements, unit u of the source's window, element
// by element into a row that may lie otherwise to the 16-byte boundaries.
template <bool BF16>
__device__ __forceinline__ void store_elems(const Window &src, const Window &dst, int u, uint4 q) {
    constexpr int E = Unit<BF16>::kElems;
    const int e0 = u * E;
    const uint32_t r[4] = {q.x, q.y, q.z, q.w};
    const int to = e0 + dst.head - src.head;
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (e0 + j >= src.head && e0 + j < src.end) {
            if constexpr (BF16)
                reinterpret_cast<uint16_t *>(dst.base)[to + j] =
                    (uint16_t)(j & 1 ? r[j / 2] >> 16 : r[j / 2]);
            else
                reinterpret_cast<uint32_t *>(dst.base)[to + j] = r[j];
        }
}

// The elements [lo, hi) of a unit that starts at element e0 of g's window, as
// far as they lie in the row.
template <bool BF16>
__device__ __forceinline__ void store_some(const Window &g, int e0, int lo, int hi,
                                           const uint4 &q) {
    constexpr int E = Unit<BF16>::kElems;
    const uint32_t r[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (j >= lo && j < hi && e0 + j >= g.head && e0 + j < g.end) {
            if constexpr (BF16)
                reinterpret_cast<uint16_t *>(g.base)[e0 + j] =
                    (uint16_t)(j & 1 ? r[j / 2] >> 16 : r[j / 2]);
            else
                reinterpret_cast<uint32_t *>(g.base)[e0 + j] = r[j];
        }
}

__device__ __forceinline__ int64_t load_index(const void *p, int64_t i, int bytes) {
    return bytes == 8 ? reinterpret_cast<const int64_t *>(p)[i]
                      : (int64_t)reinterpret_cast<const int32_t *>(p)[i];
}

// log2(e) / tau as a sum of two floats, the second positive: one float alone
// would put the same relative error, of up to 2^-24 times the exponent, on
// every small term of a row's sum, and the sums of many rows' logp would keep
// it.
struct Scale {
    float hi, lo;
};
constexpr float kLog2e = 1.44269490f, kLog2eLo = 1.3846892e-07f;  // their sum: log2(e)

// Pairs of floats in one 64-bit register: the packed fp32 instructions of
// sm_100 and later do two per lane.
typedef unsigned long long f2;
__device__ __forceinline__ f2 pair(float a, float b) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(f2 p, float &a, float &b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p));
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// 2^x; results below 2^-126 of the row's (or thread's) largest term are 0.
__device__ __forceinline__ float pow2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}

// exp((x - m) / tau).  The difference comes first: a product of the type's
// lowest value and the scale would leave the range.
__device__ __forceinline__ float exp_of(float x, float m, Scale s) {
    const float d = x - m;
    return pow2(fmaf(d, s.hi, d * s.lo));
}
// ex2.approx lies below 2^x by 5.0e-8 of it on average (measured over 10^6
// arguments in [-24, 0]; exact at whole numbers).  In the sums of many rows'
// logp that would add up, so a part's sum and the factors that bring parts to
// one maximum are raised by as much: a factor of 1 stays 1, and the part's
// largest term, which is exactly 1, is left out.
constexpr float kPow2Low = 5.0e-8f;
__device__ __forceinline__ float factor_of(float m, float to, Scale s) {
    const float f = exp_of(m, to, s);
    return fmaf(f, kPow2Low, f);
}
__device__ __forceinline__ float raised(float sum) { return fmaf(sum - 1.f, kPow2Low, sum); }
__device__ __forceinline__ f2 exp_of2(f2 x, f2 neg_m, f2 hi, f2 lo) {
    const f2 d = add2(x, neg_m);
    float a, b;
    split(fma2(d, hi, mul2(d, lo)), a, b);
    return pair(pow2(a), pow2(b));
}

// A 16-byte unit of pairs, rounded to the type.
template <bool BF16>
__device__ __forceinline__ uint4 narrow(const f2 (&v)[Unit<BF16>::kElems / 2]) {
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < Unit<BF16>::kElems / 2; ++j) {
        float a, b;
        split(v[j], a, b);
        if constexpr (BF16) {
            r[j] = pack_bf16x2(a, b);
        } else {
            r[2 * j] = __float_as_uint(a);
            r[2 * j + 1] = __float_as_uint(b);
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// The pairs of a 16-byte unit.
template <bool BF16>
__device__ __forceinline__ void widen(const uint4 &q, f2 (&o)[Unit<BF16>::kElems / 2]) {
    if constexpr (BF16) {
        o[0] = pair(bf16_lo(q.x), bf16_hi(q.x));
        o[1] = pair(bf16_lo(q.y), bf16_hi(q.y));
        o[2] = pair(bf16_lo(q.z), bf16_hi(q.z));
        o[3] = pair(bf16_lo(q.w), bf16_hi(q.w));
    } else {
        o[0] = pair(__uint_as_float(q.x), __uint_as_float(q.y));
        o[1] = pair(__uint_as_float(q.z), __uint_as_float(q.w));
    }
}

// The maximum of N units.  NaN is left to the exponentials, which keep it.
template <bool BF16, int N>
__device__ __forceinline__ float max_of(const uint4 *q) {
    if constexpr (BF16) {
        __nv_bfloat162 m2 = __floats2bfloat162_rn(-INFINITY, -INFINITY);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t w[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                m2 = __hmax2(m2, *reinterpret_cast<const __nv_bfloat162 *>(&w[j]));
        }
        return fmaxf(__low2float(m2), __high2float(m2));
    } else {
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < N; ++k)
            m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(q[k].x), __uint_as_float(q[k].y))),
                      fmaxf(__uint_as_float(q[k].z), __uint_as_float(q[k].w)));
        return m;
    }
}

// The sum of exp((x - base) / tau) over N units, and with HOLD the terms.
template <bool BF16, int N, bool HOLD>
__device__ __forceinline__ float exps_of(const uint4 *q, f2 (*v)[Unit<BF16>::kElems / 2],
                                         float base, f2 hi, f2 lo) {
    constexpr int P = Unit<BF16>::kElems / 2;
    const f2 neg = pair(-base, -base);
    f2 sums[4] = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        f2 e[P];
        widen<BF16>(q[k], e);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            e[j] = exp_of2(e[j], neg, hi, lo);
            f2 &to = sums[(k * P + j) & 3];
            to = add2(to, e[j]);
            if constexpr (HOLD) v[k][j] = e[j];
        }
    }
    float a, b;
    split(add2(add2(sums[0], sums[1]), add2(sums[2], sums[3])), a, b);
    return a + b;
}

// Base of the exponentials of a part whose maximum is m (a part of nothing but
// -inf, or of nothing, has the sum 0 whatever the base).
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

// The maximum and the sum of n <= 32 parts in shared memory: (m, s) with s
// counting exp((x - m) / tau); a part of nothing is (-inf, 0).
__device__ __forceinline__ float2 join_parts(const float2 *parts, int n, int lane, Scale scale) {
    const float2 mine = lane < n ? parts[lane] : make_float2(-INFINITY, 0.f);
    const float m = warp_max(mine.x);
    return make_float2(m, warp_sum(mine.y * factor_of(mine.x, base_of(m), scale)));
}

// -------------------------------------------------------------- row kernel

// The part of a row's units that CTA `rank` of a cluster holds, `per` at most.
struct Part {
    int first, count;
};
__device__ __forceinline__ Part part_of(int units, int rank, int per) {
    const int first = min(rank * per, units);
    return {first, min(per, units - first)};
}

// The units at a row's ends that are not whole: lanes 0..E-1 of a warp stand
// for the first unit's places, E..2E-1 for the last's.
template <bool BF16>
struct Ends {
    static constexpr int E = Unit<BF16>::kElems;
    bool cut_first, cut_last;
    bool mine, inside;    // this lane's place is in such a unit; and in the row
    int unit, element;    // its unit and place in the window
    __device__ __forceinline__ Ends(const Window &w, int lane) {
        cut_first = w.head > 0 || w.end < E;
        cut_last = w.end < w.units * E && w.units > 1;
        mine = lane < 2 * E && (lane < E ? cut_first : cut_last);
        unit = lane < E ? 0 : w.units - 1;
        element = unit * E + (lane & (E - 1));
        inside = element >= w.head && element < w.end;
    }
};

// Zeros in a part of a gradient row, by one warp: whole units as bulk copies of
// `bytes` zeros in shared memory, the ends element by element.
template <bool BF16>
__device__ __forceinline__ void zero_part(const Window &w, const Part &p, int lane,
                                          const unsigned char *zeros, int bytes) {
    constexpr int E = Unit<BF16>::kElems;
    const int lo = max(p.first, (w.head + E - 1) / E), hi = min(p.first + p.count, w.end / E);
    if (lane == 0) {
        for (int64_t at = (int64_t)lo * 16; at < (int64_t)hi * 16; at += bytes)
            bulk_store(w.base + at, smem_addr(zeros),
                       (uint32_t)min((int64_t)bytes, (int64_t)hi * 16 - at));
        bulk_commit();
    }
    const Ends<BF16> ends(w, lane);
    if (ends.mine && ends.inside && ends.unit >= p.first && ends.unit < p.first + p.count)
        store1<BF16>(w.base, ends.element, 0.f);
}

constexpr int kMaxStages = 16;   // slots of a ring
constexpr int kMaxCluster = 8;
constexpr int kBatch = 32;       // rows whose scalars are fetched together

// A place in a ring of `n` slots whose mbarriers change phase with every turn.
struct Place {
    int i = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int n) {
        if (++i == n) {
            i = 0;
            phase ^= 1;
        }
    }
};

// What the consumers take of a row besides its logits: the producer's lanes
// work it out, each for a row of its own.
struct __align__(16) RowInfo {
    float4 f;      // weight, old, ref, advantage
    char *g;       // the gradient's window
    int head;      // elements before the row in the logits' window
    int g_head;    // and in the gradient's
    int target;    // < 0: the row takes no part
    float xt;      // the token's logit; NaN for a token beyond the vocabulary
};

// A sum in fp32 and what its additions rounded away (an fp64 sum in a thread
// that all the others wait for costs more).
struct Sum {
    float s, rest;
    __device__ __forceinline__ void add(float x) {
        const float t = s + x, b = t - s;
        rest += (s - (t - b)) + (x - b);
        s = t;
    }
    // (an infinite sum has no rest)
    __device__ __forceinline__ float value() const { return fabsf(s) <= FLT_MAX ? s + rest : s; }
};

__device__ __forceinline__ int clamp_count(int n, int most) { return max(0, min(n, most)); }

// The units first, first + step, ... below end that a thread holds of `count`
// consecutive ones: the block's threads in turn, or, where the gradient's row
// lies otherwise to the 16-byte boundaries, a stretch of consecutive ones for
// each warp, so that a unit's neighbour is in the next lane.
struct Units {
    int first, step, end;
};
template <int THREADS>
__device__ __forceinline__ Units units_of(int count, int tid, bool shifted) {
    if (!shifted) return {tid, THREADS, count};
    const int per = (count + THREADS - 1) / THREADS * 32, from = (tid >> 5) * per;
    return {from + (tid & 31), 32, min(count, from + per)};
}

// A unit's gradient entries from its exponentials: each times f, and k more at
// place `at` (outside [0, E): not here).
template <bool BF16>
__device__ __forceinline__ void entries(f2 (&v)[Unit<BF16>::kElems / 2], float k, f2 f, int at) {
    constexpr int E = Unit<BF16>::kElems;
#pragma unroll
    for (int h = 0; h < E / 2; ++h) v[h] = mul2(v[h], f);
    if ((unsigned)at < E) {
#pragma unroll
        for (int h = 0; h < E / 2; ++h)
            v[h] = add2(v[h], pair(at == 2 * h ? k : 0.f, at == 2 * h + 1 ? k : 0.f));
    }
}

// Store the gradient entries of a thread's units, of a part of `count` that
// starts at the window's unit u0 (k, f, at: see entries(); at counts from the
// part's start), into a row that lies to the 16-byte boundaries as its source does: whole units in
// one piece, those at the row's ends element by element.
template <bool BF16, int N, int THREADS>
__device__ __forceinline__ void store_alike(f2 (*v)[Unit<BF16>::kElems / 2], const Window &x,
                                            char *base, int u0, int count, int tid, float k, f2 f,
                                            int at) {
    constexpr int E = Unit<BF16>::kElems;
    const int left = count - tid;
    uint4 *const to = reinterpret_cast<uint4 *>(base) + u0 + tid;
    const int own = at - tid * E;
    if (x.head == 0 && (x.end & (E - 1)) == 0) {  // nothing but whole units
#pragma unroll
        for (int j = 0; j < N; ++j) {
            entries<BF16>(v[j], k, f, own - j * THREADS * E);
            if (j * THREADS < left) __stcs(to + j * THREADS, narrow<BF16>(v[j]));
        }
        return;
    }
    const Window dst = {base, x.head, x.end, x.units};
    const int lo = max((x.head + E - 1) / E - u0, 0) - tid;
    const unsigned whole = max(min(x.end / E - u0, count) - tid - lo, 0);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        entries<BF16>(v[j], k, f, own - j * THREADS * E);
        const uint4 q = narrow<BF16>(v[j]);
        if ((unsigned)(j * THREADS - lo) < whole)
            __stcs(to + j * THREADS, q);
        else if (j * THREADS < left)
            store_elems<BF16>(x, dst, u0 + j * THREADS + tid, q);
    }
}

// Store a stretch of n consecutive units, the window's unit u0 and on, lane i
// holding i, i + 32, ..., into a row g that lies otherwise to the boundaries: a
// unit of g is the end of one unit of the source and the start of the next,
// which the neighbouring lane holds.  What the stretch has only a part of goes
// out element by element.
template <bool BF16, int N>
__device__ __forceinline__ void store_shifted(f2 (*v)[Unit<BF16>::kElems / 2],
                                              const Window &x, const Window &g, int u0, int n,
                                              int lane, float k, f2 f, int at) {
    constexpr int E = Unit<BF16>::kElems;
    const int by = g.head - x.head, shift = by < 0 ? by + E : by;  // 1..E - 1 elements
    uint4 last = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (j * 32 >= n) break;
        const int i = j * 32 + lane;
        entries<BF16>(v[j], k, f, at - i * E);
        const uint4 cur = narrow<BF16>(v[j]);
        uint4 prev = lane == 31 ? last : cur;
        prev.x = __shfl_sync(0xffffffffu, prev.x, (lane + 31) & 31);
        prev.y = __shfl_sync(0xffffffffu, prev.y, (lane + 31) & 31);
        prev.z = __shfl_sync(0xffffffffu, prev.z, (lane + 31) & 31);
        prev.w = __shfl_sync(0xffffffffu, prev.w, (lane + 31) & 31);
        last = cur;
        if (i >= n) continue;
        const int e0 = (u0 + i - (by < 0)) * E;  // of the unit in g that cur starts in
        if (i > 0 && e0 >= g.head && e0 + E <= g.end)
            __stcs(reinterpret_cast<uint4 *>(g.base) + e0 / E,
                   join_units(prev, cur, shift * Unit<BF16>::kSize));
        else
            store_some<BF16>(g, e0, i > 0 ? 0 : shift,
                             E, join_units(prev, cur, shift * Unit<BF16>::kSize));
        if (i == n - 1)
            store_some<BF16>(g, e0 + E, 0, shift,
                             join_units(cur, cur, shift * Unit<BF16>::kSize));
    }
}

// Barrier 1: the consumers.
template <int THREADS>
__device__ __forceinline__ void sync_threads() {
    asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
}

// Whether every consumer says yes.
template <int THREADS>
__device__ __forceinline__ bool all_of(bool yes) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, 1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)yes), "n"(THREADS)
        : "memory");
    return r != 0;
}

// The row at a place of the kernel's order.  The gradients of the preference
// loss go from the last row to the first, so that they meet the logits that L2
// still holds of the pass before.
template <int MODE>
__device__ __forceinline__ int64_t row_at(const LogitsArgs &a, int64_t place) {
    return is_grad(MODE) ? a.n - 1 - place : place;
}

// NaN in a row that the block has given up.
template <int MODE>
__device__ __forceinline__ void give_up(const LogitsArgs &a, int64_t row) {
    a.logp[row_at<MODE>(a, row)] = NAN;
    if constexpr (MODE == kPref) {
        a.stats[row] = make_float2(NAN, NAN);
        a.coef[row] = 0.f;
    }
}

__device__ __forceinline__ Marks marks_of(const LogitsArgs &a, int clusters) {
    return {reinterpret_cast<char *>(&a.parts->mark), (int)sizeof(PolicyPart), clusters, a.claim,
            a.mark};
}
// Whether this cluster, by the consumers of its first CTA, is the one that
// finishes a small call (aloco_marks.cuh).  A second kernel for that takes 3 us of
// the host's time, which such calls are made of (48 rows of 32000: 29 -> 24 us).
// A large call has the second kernel, which the next call overlaps (8 x 1023 x
// 32000 bf16: 162 us, 167 in one kernel).  (Not inlined: the row kernel's
// registers are the rows'.)
template <int THREADS>
__device__ __noinline__ bool finishes(const LogitsArgs &a, int cluster, int clusters, int tid) {
    return last_to_come<THREADS>(marks_of(a, clusters), cluster, tid,
                                 [] { sync_threads<THREADS>(); },
                                 [](bool b) { return all_of<THREADS>(b); });
}

// Sums of up to 32 lanes, in every lane.
__device__ __forceinline__ void sum_over_warp(Sum &s) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const float x = __shfl_xor_sync(0xffffffffu, s.s, off);
        const float y = __shfl_xor_sync(0xffffffffu, s.rest, off);
        s.add(x);
        s.rest += y;
    }
}

// The policy loss's sums from the clusters' parts, by THREADS threads (barrier
// 1), in a fixed order.
template <int THREADS>
__device__ __noinline__ void add_parts(const LogitsArgs &a, int clusters, int tid,
                                          float2 (*sh)[THREADS / 32]) {
    constexpr int WARPS = THREADS / 32;
    Sum s[kTerms] = {};
    for (int c = tid; c < clusters; c += THREADS) {
        const PolicyPart *p = a.parts + c;
        const float t[kTerms] = {__ldcg(&p->term[0]), __ldcg(&p->term[1]), __ldcg(&p->term[2])};
        for (int j = 0; j < kTerms; ++j) s[j].add(t[j]);
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < kTerms; ++j) {
        sum_over_warp(s[j]);
        if ((tid & 31) == 0) sh[j][tid >> 5] = make_float2(s[j].s, s[j].rest);
    }
    sync_threads<THREADS>();
    if (tid >= 32) return;
#pragma unroll
    for (int j = 0; j < kTerms; ++j) {
        s[j] = {0.f, 0.f};
        if (tid < WARPS) {
            s[j].s = sh[j][tid].x;
            s[j].rest = sh[j][tid].y;
        }
        sum_over_warp(s[j]);
    }
    if (tid == 0) {
        const float gain = s[0].value(), kl = s[1].value();
        // (without a coefficient the KL sum is only watched, and may be infinite)
        a.terms_out[0] = a.kl != 0.f ? fmaf(a.kl, kl, gain) : gain;
        a.terms_out[1] = gain;
        a.terms_out[2] = kl;
        a.terms_out[3] = s[2].value();
    }
}

// ---------------------------------------------------- pairs of log ratios

// In fp32 with the additions' rests kept: fp64 units are rare here (one fp64 exp
// took longer than a pair's rows).  THREADS threads, which barrier 1 counts.
constexpr int kPairBlock = 512;

// The sums of N values over the threads in a fixed order, in every thread.
template <int THREADS, int N>
__device__ __forceinline__ void block_totals(Sum (&v)[N], int tid, float2 (*sh)[THREADS / 32]) {
    const int lane = tid & 31;
    sync_threads<THREADS>();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        sum_over_warp(v[i]);
        if (lane == 0) sh[i][tid >> 5] = make_float2(v[i].s, v[i].rest);
    }
    sync_threads<THREADS>();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = {0.f, 0.f};
        if (lane < THREADS / 32) {
            v[i].s = sh[i][lane].x;
            v[i].rest = sh[i][lane].y;
        }
        sum_over_warp(v[i]);
    }
}

// -(1 - eps) log sigmoid(z) - eps log sigmoid(-z)
__device__ __forceinline__ float pair_loss(float z, float eps) {
    // -log sigmoid(z) = log(1 + exp(-|z|)) + max(-z, 0); a margin of +inf costs
    // nothing where no labels are flipped (0 * inf is NaN)
    return log1pf(expf(-fabsf(z))) +
           (z < 0.f ? (1.f - eps) * -z : eps == 0.f && z == INFINITY ? 0.f : eps * z);
}

// Log ratios of pair k and the coefficients of its rows.
template <int THREADS>
__device__ __forceinline__ void one_pair(const LogitsArgs &a, int64_t k, int tid,
                                         float2 (*sh)[THREADS / 32]) {
    int64_t cu[3];
    for (int i = 0; i < 3; ++i) {
        cu[i] = load_index(a.cu, 2 * k + i, a.cu_bytes);
        cu[i] = cu[i] < 0 ? 0 : cu[i] > a.n ? a.n : cu[i];
    }
    Sum s[2] = {};
#pragma unroll 2
    for (int64_t r = cu[0] + tid; r < cu[2]; r += THREADS) {
        const bool live = load_index(a.target, r, a.target_bytes) >= 0;
        const float lp = __ldcg(a.logp + r), ref = a.ref ? a.ref[r] : 0.f;
        if (live && r < cu[1]) {
            s[0].add(lp);
            s[0].add(-ref);
        } else if (live) {
            s[1].add(lp);
            s[1].add(-ref);
        }
    }
    block_totals<THREADS>(s, tid, sh);
    const float chosen = s[0].value(), rejected = s[1].value();
    if (tid == 0) {
        a.ratios[2 * k] = chosen;
        a.ratios[2 * k + 1] = rejected;
    }
    if (!a.g.data) return;
    const float z = a.beta * (chosen - rejected), t = expf(-fabsf(z));
    // sigmoid(z) - 1 + eps, without the difference where z is large
    const float slope =
        (z >= 0.f ? a.eps - t / (1.f + t) : t / (1.f + t) - (1.f - a.eps)) * a.per_pair;
    for (int64_t r = cu[0] + tid; r < cu[2]; r += THREADS)
        if (load_index(a.target, r, a.target_bytes) >= 0) a.coef[r] = r < cu[1] ? slope : -slope;
}

// The loss, from the ratios that are in memory.
template <int THREADS>
__device__ __forceinline__ void mean_of_pairs(const LogitsArgs &a, int tid,
                                              float2 (*sh)[THREADS / 32]) {
    sync_threads<THREADS>();
    Sum s[1] = {};
    for (int64_t k = tid; k < a.pairs; k += THREADS)
        s[0].add(pair_loss(a.beta * (__ldcg(a.ratios + 2 * k) - __ldcg(a.ratios + 2 * k + 1)), a.eps));
    block_totals<THREADS>(s, tid, sh);
    if (tid == 0) a.loss[0] = a.pairs ? s[0].value() / (float)a.pairs : 0.f;
}

// All pairs, by the consumers of the last block to come.
template <int THREADS>
__device__ __noinline__ void all_pairs(const LogitsArgs &a, int tid, float2 (*sh)[THREADS / 32]) {
    for (int64_t k = 0; k < a.pairs; ++k) one_pair<THREADS>(a, k, tid, sh);
    mean_of_pairs<THREADS>(a, tid, sh);
}

// Testing only: whether block 0 leaves out the copy of its slot number `slot`;
// the first one may come late.  Where it is too late for its row, that row's
// log-probability is 0 until the copy has landed.
template <int MODE>
__device__ __noinline__ bool stalls(const LogitsArgs &a, unsigned slot) {
    if (a.test_stall1 < 0 && slot == 0) {
        for (const long long t0 = clock64(); clock64() - t0 < -a.test_stall1;) {}
        a.logp[row_at<MODE>(a, 0)] = 0.f;
    }
    return slot + 1 == a.test_stall1;
}

// Wait, by the producer's warp, for the last copies into a ring whose slots were
// armed `filled` times.
template <int MODE>
__device__ __noinline__ void land(const LogitsArgs &a, const uint64_t *full, unsigned filled,
                                  int stages) {
    bool landed = true;
    for (unsigned k = filled > (unsigned)stages ? filled - stages : 0; k < filled; ++k)
        landed &= mbar_wait(smem_addr(full + k % stages), k / stages & 1, nullptr);
    if (a.test_stall1 < 0 && !blockIdx.x && landed) a.logp[row_at<MODE>(a, 0)] = NAN;  // see stalls
}

// THREADS consumers and one producer warp.  CTA c of a cluster holds its part
// of a row in the registers of its consumers: thread t the units k * THREADS +
// t of the part, k < UPT.  A slot of the ring is DEPTH units of every thread.
template <bool BF16, int THREADS, int UPT, int DEPTH, int CTAS, int MODE>
__global__ void __launch_bounds__(THREADS + 32, CTAS)
    row_kernel(const __grid_constant__ LogitsArgs a) {
    constexpr int E = Unit<BF16>::kElems, P = E / 2;
    constexpr int WARPS = THREADS / 32;
    constexpr int SLOT = DEPTH * THREADS;          // units of a slot
    constexpr int ZEROS = SLOT * 16 / 4 < 8192 ? SLOT * 16 / 4 : 8192;  // bytes
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_joined[2];
    __shared__ __align__(8) uint64_t s_rows_full[2], s_rows_empty[2];
    __shared__ RowInfo s_rows[2][kBatch];
    __shared__ float2 s_warp[2][WARPS];
    __shared__ float2 s_sums[is_policy(MODE) ? kTerms : MODE == kPref ? 2 : 1][WARPS];
    __shared__ __align__(8) float2 s_cta[2][kMaxCluster];
    __shared__ volatile int s_abort, s_bad[2];
    __shared__ unsigned s_filled;

    const cg::cluster_group cluster = cg::this_cluster();
    const int C = a.cluster, rank = (int)(blockIdx.x % (unsigned)C);
    const int64_t step = gridDim.x / (unsigned)C;
    const int64_t row0 = blockIdx.x / (unsigned)C;
    const int tid = threadIdx.x, lane = tid & 31;
    const int stages = a.stages;
    const volatile int *const aborted = &s_abort;
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(smem_addr(&s_full[i]), 1);
            mbar_init(smem_addr(&s_empty[i]), WARPS);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&s_joined[i]), 1);
            mbar_init(smem_addr(&s_rows_full[i]), 1);
            mbar_init(smem_addr(&s_rows_empty[i]), WARPS);
        }
        s_abort = s_bad[0] = s_bad[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (C > 1)
        cluster.sync();
    else
        __syncthreads();
    wait_for_previous();
    if (MODE == kPref && !a.finish && blockIdx.x == 0 && tid == 0) *a.ticket = 0;

    if (tid >= THREADS) {
        // Producer: the rows' scalars, kBatch rows at a time, and their parts,
        // slot after slot, as far ahead as the ring is free.  Whole units come
        // as bulk copies; the elements of a unit at a row's end that is not
        // whole come one by one, with -inf beside them.
        Place place, batch;
        unsigned filled = 0;
        bool ok = true, again = false;
        unsigned mixed = 0;  // slots that hold stores of this warp's
        const bool tested = a.test_stall1 != 0 && blockIdx.x == 0;
        unsigned char *const zeros = ring + (size_t)stages * SLOT * 16;
        if (writes_grad(MODE) && a.g.data) {
            for (int i = lane; i < ZEROS / 16; i += 32)
                reinterpret_cast<uint4 *>(zeros)[i] = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
        }
        for (int64_t base = row0; base < a.n && ok; base += kBatch * step, batch.next(2)) {
            const int64_t my_place = base + lane * step;
            const int64_t my_row = row_at<MODE>(a, my_place);
            RowInfo mine = {make_float4(1.f, 0.f, 0.f, 0.f), nullptr, 0, 0, -1, NAN};
            Window my_x = {};
            int64_t t = -1;
            if (my_place < a.n) {
                t = load_index(a.target, my_row, a.target_bytes);
                if constexpr (is_policy(MODE)) {
                    mine.f = make_float4(a.w[my_row], a.old[my_row], a.ref ? a.ref[my_row] : 0.f,
                                         a.adv[my_row]);
                    if (mine.f.x == 0.f) t = -1;
                }
                if constexpr (is_grad(MODE)) {
                    const float k = a.coef[my_row] * a.inv_temp;
                    const float2 q = a.stats[my_row];
                    mine.f = make_float4(k, -k * q.y, base_of(q.x), 0.f);
                    if (k == 0.f) t = -1;
                }
                if (writes_grad(MODE) && a.g.data) {
                    const Window g = window_of<BF16>(a.g, my_row, a.vocab);
                    mine.g = g.base;
                    mine.g_head = g.head;
                }
                my_x = window_of<BF16>(a.x, my_row, a.vocab);
                mine.head = my_x.head;
            }
            // read here, and so before this CTA lets the row's gradient be
            // written, which may lie over the logits
            if (!is_grad(MODE) && t >= 0 && t < a.vocab) mine.xt = load1<BF16>(my_x.base, my_x.head + (int)t);
            mine.target = t < 0 ? -1 : t >= a.vocab ? a.vocab : (int)t;
            unsigned todo = __ballot_sync(0xffffffffu, t >= 0);
            // rows without a part to play: this CTA's part of their zeros
            unsigned idle = writes_grad(MODE) && a.g.data
                                ? __ballot_sync(0xffffffffu, my_place < a.n && t < 0) : 0u;
            // The window of the next row and the elements at its ends are
            // fetched a row ahead.
            Window ahead_x = {};
            float ahead_edge = 0.f;
            const auto look_ahead = [&](int from) {
                ahead_x = window_at<BF16>(
                    reinterpret_cast<char *>(__shfl_sync(
                        0xffffffffu, reinterpret_cast<uint64_t>(my_x.base), from)),
                    __shfl_sync(0xffffffffu, my_x.head, from), a.vocab);
                const Ends<BF16> ends(ahead_x, lane);
                ahead_edge = ends.mine && ends.inside ? load1<BF16>(ahead_x.base, ends.element)
                                                      : -INFINITY;
            };
            if (todo) look_ahead(__ffs(todo) - 1);
            // The scalars go out behind the first row's copies, which then do
            // not wait for them; ahead of them where a part may be longer than
            // the ring, which only consumers that know the row make room in.
            bool told = false;
            const auto tell = [&] {
                told = true;
                if (again)
                    ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&s_rows_empty[batch.i]),
                                                           batch.phase ^ 1, aborted));
                if (!ok) return;
                s_rows[batch.i][lane] = mine;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&s_rows_full[batch.i]));
            };
            if (!is_policy(MODE)) tell();
            while (ok && (!told || todo || idle)) {
                if (idle && (!todo || (told && __ffs(idle) < __ffs(todo)))) {
                    const int from = __ffs(idle) - 1;
                    idle &= idle - 1;
                    const Window g = window_at<BF16>(
                        reinterpret_cast<char *>(__shfl_sync(
                            0xffffffffu, reinterpret_cast<uint64_t>(mine.g), from)),
                        __shfl_sync(0xffffffffu, mine.g_head, from), a.vocab);
                    zero_part<BF16>(g, part_of(g.units, rank, a.per), lane, zeros, ZEROS);
                } else if (todo) {
                    todo &= todo - 1;
                    const Window x = ahead_x;
                    const float edge = ahead_edge;
                    if (todo) look_ahead(__ffs(todo) - 1);
                    const Part p = part_of(x.units, rank, a.per);
                    const Ends<BF16> ends(x, lane);
                    for (int s = 0; s < p.count; s += SLOT) {
                        const uint32_t full = smem_addr(&s_full[place.i]);
                        unsigned char *at = ring + (size_t)place.i * SLOT * 16;
                        if (filled >= (unsigned)stages)
                            ok = __all_sync(0xffffffffu,
                                            mbar_wait(smem_addr(&s_empty[place.i]),
                                                      place.phase ^ 1, aborted));
                        if (!ok) break;
                        // earlier stores to this slot come before its next copy
                        if (mixed >> place.i & 1) {
                            fence_proxy_async_smem();
                            mixed &= ~(1u << place.i);
                        }
                        int lo = p.first + s, hi = p.first + min(s + SLOT, p.count);
                        const int u0 = lo;
                        if (ends.mine && ends.unit >= lo && ends.unit < hi)
                            store1<BF16>((char *)at, ends.element - u0 * E, edge);
                        const bool cut_lo = ends.cut_first && lo == 0;
                        const bool cut_hi = ends.cut_last && hi == x.units;
                        if (cut_lo || cut_hi) mixed |= 1u << place.i;
                        lo += cut_lo;
                        hi -= cut_hi;
                        __syncwarp();
                        if (lane == 0) {
                            const uint32_t bytes = hi > lo ? (uint32_t)(hi - lo) * 16 : 0;
                            mbar_arrive_expect_tx(full, bytes);
                            if (bytes && !(tested && stalls<MODE>(a, filled)))
                                bulk_load(smem_addr(at + (size_t)(lo - u0) * 16),
                                          x.base + (size_t)lo * 16, bytes, full);
                        }
                        place.next(stages);
                        ++filled;
                    }
                }
                if (!told && ok) tell();
            }
            again = again || batch.i == 1;
        }
        // the zeros' source stays until their copies have read it
        if (writes_grad(MODE) && lane == 0) bulk_wait_all();
        if (!ok) s_abort = 1;
        s_filled = filled;
    } else {
        const Scale scale = {a.scale, a.scale_lo};
        const f2 hi2 = pair(scale.hi, scale.hi), lo2 = pair(scale.lo, scale.lo);
        Place place, batch;
        unsigned rows = 0;  // rows taken
        bool ok = true;
        int next = 0;       // the row's place in its batch
        Sum terms[kTerms] = {};
        // All consumers leave together where a wait of one of them ran out: NaN
        // in this row and the block's later ones, and no barrier armed again.
        const auto leave = [&](int64_t row) {
            s_abort = 1;
            for (; row < a.n; row += step)
                if (rank == 0 && tid == 0) give_up<MODE>(a, row);
            terms[0].s = terms[1].s = NAN;
        };
        // This thread's units of the next slot, which holds `count` (none: 0),
        // -inf where it has none.
        const auto take_slot = [&](uint4 *q, int count, bool shifted) {
            const Units w = units_of<THREADS>(count, tid, may_shift(MODE) && shifted);
            const int left = w.end - w.first;
            bool here = true;
            if (count > 0)
                here = __all_sync(0xffffffffu, mbar_wait(smem_addr(&s_full[place.i]), place.phase,
                                                         aborted));
            const uint4 *slot = reinterpret_cast<const uint4 *>(ring) + (size_t)place.i * SLOT + w.first;
#pragma unroll
            for (int j = 0; j < DEPTH; ++j) {
                const uint32_t none = BF16 ? 0xff80ff80u : 0xff800000u;  // -inf
                q[j] = make_uint4(none, none, none, none);
                if (j * w.step < left) q[j] = slot[j * w.step];
            }
            if (count > 0) {
                __syncwarp();
                // A slot whose wait ran out is never given back: the producer
                // may not arm its barrier again before the copy has landed.
                // Nor is a later one, whose wait may succeed on an older phase
                // (a row that is held takes no place of the ring twice, and the
                // block leaves at its barrier).
                if constexpr (!is_policy(MODE)) here = ok = ok && here;
                if (!here)
                    s_abort = s_bad[rows & 1] = 1;
                else if (lane == 0)
                    mbar_arrive(smem_addr(&s_empty[place.i]));
                place.next(stages);
            }
        };
        for (int64_t row = row0; row < a.n; row += step) {
            if (next == kBatch) {
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&s_rows_empty[batch.i]));
                batch.next(2);
                next = 0;
            }
            if (next == 0 && !all_of<THREADS>(mbar_wait(smem_addr(&s_rows_full[batch.i]),
                                                        batch.phase, aborted))) {
                // without the rows' scalars nothing can be said of them
                leave(row);
                break;
            }
            const RowInfo r = s_rows[batch.i][next++];
            const bool first = rank == 0 && tid == 0;
            if (r.target < 0) {  // the producer writes its zeros
                if (!is_grad(MODE) && first) {
                    a.logp[row] = 0.f;
                    if constexpr (MODE == kPref) a.coef[row] = 0.f;
                }
                continue;
            }
            const Window x = window_at<BF16>(nullptr, r.head, a.vocab);
            const Part p = part_of(x.units, rank, a.per);
            if constexpr (is_grad(MODE)) {
                // the preference loss's gradient, slot by slot
                const f2 neg = pair(-r.f.z, -r.f.z);
                const int at = r.target < a.vocab ? x.head + r.target : INT_MIN / 2;
                const bool shifted = r.g_head != r.head;
                for (int u = 0; u < p.count; u += SLOT) {
                    const int count = clamp_count(p.count - u, SLOT), u0 = p.first + u;
                    uint4 q[DEPTH];
                    take_slot(q, count, shifted);
                    if (!ok && first) give_up<MODE>(a, row);
                    const float f = ok ? r.f.y : NAN;
                    f2 v[DEPTH][P];
#pragma unroll
                    for (int j = 0; j < DEPTH; ++j) {
                        widen<BF16>(q[j], v[j]);
#pragma unroll
                        for (int h = 0; h < P; ++h) v[j][h] = exp_of2(v[j][h], neg, hi2, lo2);
                    }
                    if (may_shift(MODE) && shifted) {
                        const Units w = units_of<THREADS>(count, tid, true);
                        const int from = u0 + w.first - lane;
                        store_shifted<BF16, DEPTH>(v, x, window_at<BF16>(r.g, r.g_head, a.vocab), from,
                                                   max(w.end - w.first + lane, 0), lane, r.f.x,
                                                   pair(f, f), at - from * E);
                    } else {
                        store_alike<BF16, DEPTH, THREADS>(v, x, r.g, u0, count, tid, r.f.x, pair(f, f),
                                                          at - u0 * E);
                    }
                }
                continue;
            }
            // this thread's maximum, and the sum of its exp((x - maximum) /
            // tau): all of them at once where they are kept for the gradient,
            // slot by slot otherwise
            constexpr bool kHold = is_policy(MODE);
            const bool shifted = r.g && r.g_head != r.head;
            f2 v[kHold ? UPT : 1][P];
            float mt = -INFINITY, st = 0.f;
            if constexpr (kHold) {
                uint4 q[UPT];
#pragma unroll
                for (int k = 0; k < UPT; k += DEPTH)
                    take_slot(q + k, clamp_count(p.count - k * THREADS, SLOT), shifted);
                mt = max_of<BF16, UPT>(q);
                st = exps_of<BF16, UPT, true>(q, v, base_of(mt), hi2, lo2);
            } else {
                for (int u = 0; u < p.count; u += SLOT) {
                    uint4 q[DEPTH];
                    take_slot(q, clamp_count(p.count - u, SLOT), false);
                    const float before = mt;
                    mt = fmaxf(mt, max_of<BF16, DEPTH>(q));
                    st = st * factor_of(before, base_of(mt), scale) +
                         exps_of<BF16, DEPTH, false>(q, v, base_of(mt), hi2, lo2);
                }
            }

            // the row's maximum and sum: warps, CTA, cluster, each in a fixed
            // order.  Two sets of shared places take turns, so that one
            // barrier a row is enough: a CTA sends row i + 1's pair only when
            // all its warps have read row i's.  (Every warp's pair sent to
            // every CTA, without the barrier, took longer: 704 against 665 us
            // at 8000 rows of 128256 bf16.)
            const unsigned turn = rows & 1, phase = (rows >> 1) & 1;
            ++rows;
            const float mw = warp_max(mt);
            const float sw = warp_sum(raised(st) * factor_of(mt, base_of(mw), scale));
            if (lane == 0) s_warp[turn][tid >> 5] = make_float2(mw, sw);
            asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
            if (s_bad[turn]) {  // written before this barrier only: the same for all
                leave(row);
                break;
            }
            float2 part;
            if (C == 1 || tid < 32) part = join_parts(s_warp[turn], WARPS, lane, scale);
            if (C > 1) {
                // every CTA sends its pair to all CTAs of the cluster, and
                // waits for theirs
                const uint32_t bar = smem_addr(&s_joined[turn]);
                if (tid == 0) mbar_arrive_expect_tx(bar, C * 8);
                if (tid < C) {
                    uint32_t to, there;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                                 : "=r"(to) : "r"(smem_addr(&s_cta[turn][rank])), "r"(tid));
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                                 : "=r"(there) : "r"(bar), "r"(tid));
                    asm volatile(
                        "st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 "
                        "[%0], {%1, %2}, [%3];" ::"r"(to), "f"(part.x), "f"(part.y), "r"(there)
                        : "memory");
                }
                // (where that runs out, this row is NaN and the next one's
                // barrier is where the block leaves)
                const bool here = __all_sync(0xffffffffu, mbar_wait(bar, phase, aborted));
                part = join_parts(s_cta[turn], C, lane, scale);
                if (!here) {
                    s_abort = s_bad[turn ^ 1] = 1;
                    part.y = NAN;
                }
            }
            const float m = part.x, z = part.y;
            // a row without a finite logit leaves z = 0: -inf - -inf
            const float logp = z > 0.f ? fmaf(r.xt - m, a.inv_temp, -logf(z)) : NAN;

            if constexpr (is_policy(MODE)) {
                const float weight = r.f.x;
                const Scale unit = {kLog2e, kLog2eLo};
                const float ratio = exp_of(logp, r.f.y, unit);
                // (a ratio beyond fp32 of a finite logarithm is no infinity: without
                // an advantage it counts 0)
                const float free = r.f.w == 0.f && ratio == INFINITY && r.f.y >= -FLT_MAX
                                       ? 0.f : ratio * r.f.w;
                const float bound = fminf(fmaxf(ratio, a.lo), a.hi) * r.f.w;
                const bool act = free <= bound;
                const float d = r.f.z - logp;
                const float back = exp_of(r.f.z, logp, unit);
                if (first) {
                    a.logp[row] = logp;
                    terms[0].add(-weight * (act || free != free ? free : bound));
                    if (a.ref) terms[1].add(weight * (expm1f(d) - d));
                    if (!act) terms[2].add(weight);
                }
                if (!r.g) continue;
                const float k =
                    weight * ((a.kl != 0.f ? a.kl * (1.f - back) : 0.f) -
                              (act || free != free ? free : 0.f)) * a.inv_temp;
                // this thread's values are exp((x - base) / tau), all 0 where
                // it has no finite logit
                const float f = -k * (z > 0.f ? (mt == -INFINITY ? 0.f
                                                 : exp_of(mt, m, scale) * __fdividef(1.f, z))
                                              : NAN);
                const f2 ff = pair(f, f);
                // the token's own entry (none within reach where it is beyond
                // the vocabulary, whose rows are NaN)
                const int at = r.target < a.vocab ? x.head + r.target : INT_MIN / 2;
#pragma unroll
                for (int i = 0; i < UPT; i += DEPTH) {
                    const int count = clamp_count(p.count - i * THREADS, SLOT);
                    const int u0 = p.first + i * THREADS;
                    if (may_shift(MODE) && shifted) {
                        const Units w = units_of<THREADS>(count, tid, true);
                        const int from = u0 + w.first - lane;
                        store_shifted<BF16, DEPTH>(v + i, x, window_at<BF16>(r.g, r.g_head, a.vocab),
                                                   from, max(w.end - w.first + lane, 0), lane, k, ff,
                                                   at - from * E);
                    } else {
                        store_alike<BF16, DEPTH, THREADS>(v + i, x, r.g, u0, count, tid, k, ff,
                                                          at - u0 * E);
                    }
                }
            } else if (first) {
                a.logp[row] = logp;
                if constexpr (MODE == kPref) {
                    a.stats[row] = make_float2(m, z > 0.f ? 1.f / z : NAN);
                    a.coef[row] = 0.f;
                }
            }
        }
        // (the first CTA of a cluster has written what its rows leave)
        if constexpr (is_policy(MODE)) {
            if (rank == 0 && tid == 0) {
                PolicyPart *const p = a.parts + row0;
                for (int j = 0; j < kTerms; ++j) p->term[j] = terms[j].value();
            }
        }
        if ((MODE == kPolicySmall || MODE == kPolicyShifted || MODE == kPref) && a.finish &&
            rank == 0 && finishes<THREADS>(a, (int)row0, (int)step, tid)) {
            if constexpr (is_policy(MODE)) add_parts<THREADS>(a, (int)step, tid, s_sums);
            if constexpr (MODE == kPref) all_pairs<THREADS>(a, tid, s_sums);
            if (tid == 0) give_back(marks_of(a, (int)step));
        }
    }
    // No copy may land after the block has ended, whoever has given up: where all
    // slots were free the producer comes here without having waited, and the
    // consumers may leave while the last copies are on their way.  (Only then:
    // the producer's waiting here in every block cost 164 -> 169 us at 8 x 1023 x
    // 32000 bf16.)
    __syncthreads();
    if (s_abort && tid >= THREADS) land<MODE>(a, s_full, s_filled, stages);
    // no CTA leaves while another may still write to its memory
    if (C > 1)
        cluster.sync();
    else
        __syncthreads();
}

constexpr int kSumBlock = 256;
__global__ void __launch_bounds__(kSumBlock)
    policy_sums_kernel(const __grid_constant__ LogitsArgs a, int clusters) {
    __shared__ float2 sh[kTerms][kSumBlock / 32];
    wait_for_previous();
    add_parts<kSumBlock>(a, clusters, threadIdx.x, sh);
}

__global__ void __launch_bounds__(kPairBlock)
    pairs_kernel(const __grid_constant__ LogitsArgs a) {
    __shared__ float2 sh[2][kPairBlock / 32];
    __shared__ bool last;
    const int tid = threadIdx.x;
    wait_for_previous();
    for (int64_t k = blockIdx.x; k < a.pairs; k += gridDim.x) one_pair<kPairBlock>(a, k, tid, sh);
    if (gridDim.x > 1) {
        __threadfence();
        __syncthreads();
        if (tid == 0) last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
        __syncthreads();
        if (!last) return;
        __threadfence();
    }
    mean_of_pairs<kPairBlock>(a, tid, sh);
}

// Launch of a row kernel of THREADS consumers with EPT elements each: a
// cluster of as many CTAs as a row takes (more where there are too few rows for
// the SMs), and as many clusters as the device holds at once, which take the
// rows in turn.
template <bool BF16, int THREADS, int EPT, int DEPTH, int STAGES, int CTAS, int MODE>
cudaError_t launch_rows_as(const LogitsArgs &in, int sm_count, cudaStream_t stream, int *used) {
    constexpr int E = Unit<BF16>::kElems, UPT = EPT / E;
    constexpr int kSlot = DEPTH * THREADS * 16;
    constexpr int kSmem = STAGES * kSlot + (!writes_grad(MODE) ? 0 : kSlot / 4 < 8192 ? kSlot / 4 : 8192);
    static_assert(STAGES <= kMaxStages && UPT % DEPTH == 0, "ring");
    static PerDevice ready, most[kMaxCluster + 1];
    const auto kernel = row_kernel<BF16, THREADS, UPT, DEPTH, CTAS, MODE>;
    const int units = (in.vocab + 2 * (E - 1)) / E;
    // (the kernels that do not hold a row take a part of any length)
    int C = is_policy(MODE) ? (units + THREADS * UPT - 1) / (THREADS * UPT) : 1;
    if (C > kMaxCluster) return cudaErrorInvalidValue;
    while (C < kMaxCluster && in.n * (C + 1) <= sm_count && units >= (C + 1) * THREADS) ++C;

    const int dev = PerDevice::device();
    if (!ready.get(dev)) {
        const cudaError_t e = cudaFuncSetAttribute(
            kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        ready.set(dev, 1);
    }
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    // the kernel sets itself up while the one before it ends
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)C);
    cfg.blockDim = dim3(THREADS + 32);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = most[C].get(dev);
    if (!clusters) {
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
        if (e != cudaSuccess) return e;
        if (clusters < 1) return cudaErrorInvalidConfiguration;
        most[C].set(dev, clusters);
    }
    cfg.numAttrs = 2;
    LogitsArgs a = in;
    a.stages = STAGES;
    a.cluster = C;
    a.per = (units + C - 1) / C;
    *used = (int)(in.n < clusters ? in.n : clusters);
    cfg.gridDim = dim3((unsigned)(*used * C));
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <bool BF16, int MODE>
cudaError_t launch_rows(const LogitsArgs &a, int sm_count, cudaStream_t stream, int *used) {
    *used = 0;
    if (a.n == 0) return cudaSuccess;
    // units of a thread in a slot of the ring: a whole part in bf16; in fp32,
    // whose parts are twice as long, a sixth of it (1380 live rows of 32000: 67
    // against 73 us with half a part), but half of it where rows lie askew (3 x
    // 511 x 50257 shifted: 137 against 166 us)
    constexpr int kDeep = BF16 || MODE == kPolicyShifted ? 9 : 3;
    if (a.vocab <= 32 * 72 - 14)
        return launch_rows_as<BF16, 32, 72, 9, 3, 8, MODE>(a, sm_count, stream, used);
    if (a.vocab <= 64 * 72 - 14)
        return launch_rows_as<BF16, 64, 72, 9, 3, 5, MODE>(a, sm_count, stream, used);
    if constexpr (!is_policy(MODE)) {
        return launch_rows_as<BF16, 224, 72, 3, 4, 4, MODE>(a, sm_count, stream, used);
    } else {
        if (a.vocab <= 128 * 72 - 14)
            return launch_rows_as<BF16, 128, 72, 9, 3, 3, MODE>(a, sm_count, stream, used);
        // Two CTAs an SM or one of twice the size: the large one where it holds
        // the row alone or in two (8 x 1023 x 32000 bf16: 162 us, 198 as a
        // cluster of two small ones; x 50304: 328 as two, 335 as four), else
        // the one whose cluster the row fills better (8 x 1000 x 128256: 640
        // us at 0.99 of eight small ones, 674 at 0.93 of four; 8 x 1023 x
        // 100000: 642 us at 0.89 of seven, 574 at 0.96 of three).
        const int units = (a.vocab + 2 * (16 / (BF16 ? 2 : 4) - 1)) / (16 / (BF16 ? 2 : 4));
        constexpr int kOne = 480 * (BF16 ? 9 : 18), kTwo = 224 * (BF16 ? 9 : 18);
        const int one = (units + kOne - 1) / kOne, two = (units + kTwo - 1) / kTwo;
        if (two == 1 || (one > 2 && two <= kMaxCluster && two * kTwo < one * kOne))
            return launch_rows_as<BF16, 224, 72, kDeep, 27 / kDeep, 2, MODE>(a, sm_count, stream,
                                                                             used);
        return launch_rows_as<BF16, 480, 72, kDeep, 27 / kDeep, 1, MODE>(a, sm_count, stream, used);
    }
}

// A launch that may begin before the kernel ahead of it in the stream has
// ended: it waits for that kernel itself.
template <typename... Params, typename... Args>
cudaError_t launch_behind(void (*kernel)(Params...), unsigned grid, unsigned block,
                          cudaStream_t stream, Args... args) {
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Whether all rows of the gradient lie to the 16-byte boundaries as the logits'.
template <bool BF16>
bool rows_alike(const LogitsArgs &a) {
    if (!a.g.data) return true;
    const int64_t size = Unit<BF16>::kSize, per = a.x.per_batch;
    int64_t off = (int64_t)((uintptr_t)a.x.data - (uintptr_t)a.g.data);
    if (per > 1) off |= (a.x.row_stride - a.g.row_stride) * size;
    if (a.n > per) off |= (a.x.batch_stride - a.g.batch_stride) * size;
    return (off & 15) == 0;
}

template <bool BF16>
cudaError_t launch_policy_rows(const LogitsArgs &in, int sm_count, cudaStream_t stream) {
    LogitsArgs a = in;
    int used;
    if (a.n == 0) return cudaMemsetAsync(a.terms_out, 0, (kTerms + 1) * sizeof(float), stream);
    // about where the GPU's time passes the host's
    a.finish = a.n * a.vocab * Unit<BF16>::kSize < ((int64_t)80 << 20);
    const cudaError_t e =
        !rows_alike<BF16>(a) ? launch_rows<BF16, kPolicyShifted>(a, sm_count, stream, &used)
        : a.finish           ? launch_rows<BF16, kPolicySmall>(a, sm_count, stream, &used)
                             : launch_rows<BF16, kPolicy>(a, sm_count, stream, &used);
    if (e != cudaSuccess || a.finish) return e;
    return launch_behind(policy_sums_kernel, 1, kSumBlock, stream, a, used);
}

template <bool BF16>
cudaError_t launch_preference_rows(const LogitsArgs &in, int sm_count, cudaStream_t stream) {
    LogitsArgs a = in;
    int used;
    // few rows: the row kernel's last cluster is done with the pairs sooner than
    // another kernel is launched
    a.finish = a.n > 0 && a.n <= 2048 && a.pairs <= 16;
    cudaError_t e = launch_rows<BF16, kPref>(a, sm_count, stream, &used);
    if (e == cudaSuccess && !a.finish) {
        const unsigned blocks =
            a.n == 0 || a.pairs < 2 ? 1u : (unsigned)(a.pairs < 1024 ? a.pairs : 1024);
        e = launch_behind(pairs_kernel, blocks, kPairBlock, stream, a);
    }
    if (e != cudaSuccess || !a.g.data) return e;
    a.test_stall1 = 0;
    return rows_alike<BF16>(a) ? launch_rows<BF16, kGrad>(a, sm_count, stream, &used)
                               : launch_rows<BF16, kGradShifted>(a, sm_count, stream, &used);
}

}  // namespace

}  // namespace aloco
