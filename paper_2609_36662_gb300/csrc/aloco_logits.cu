// Log-probabilities of tokens, and the policy and preference losses with their
// gradients by the logits.
//
// A row x[0..V) with its token a and temperature tau:
//   m = max x,  z = sum_j exp((x_j - m) / tau),
//   logp = (x_a - m) / tau - log z,   p_j = exp((x_j - m) / tau) / z
//   dL/dx_j = k ([j = a] - p_j),  k = dL/dlogp / tau.
//
// Row kernel: a cluster of C CTAs holds a row in its registers, 16-byte units
// of it in a fixed pattern per thread.  Every thread turns its elements into
// exp((x - own maximum) / tau) once; one reduction over (maximum, sum) pairs
// (warp, CTA, and through distributed shared memory the cluster) gives m and
// z, and the gradient is each kept value times one factor per thread.  The
// logits are thus read once and the gradient written once.
// The preference loss needs every row of a pair before any of its gradients:
// its first kernel leaves m and 1/z of every row, its second adds the log
// ratios, and its third reads the logits again.
//
// A row may start off a 16-byte boundary (odd vocabularies): the units are
// those of the aligned window around it, and the two at its ends are read and
// written element by element.
#include <cooperative_groups.h>

#include "aloco_logits.h"
#include "aloco_sync_kernel.cuh"

namespace aloco {

namespace {

namespace cg = cooperative_groups;

constexpr int kFwd = 0, kPolicy = 1, kPref = 2;  // what a row kernel leaves

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
__device__ __forceinline__ Window window_of(const Rows &r, int64_t row, int vocab) {
    const int64_t b = row / r.per_batch;
    char *p = r.data + (b * r.batch_stride + (row - b * r.per_batch) * r.row_stride) *
                           Unit<BF16>::kSize;
    Window w;
    const int off = (int)((uintptr_t)p & 15);
    w.base = p - off;
    w.head = off / Unit<BF16>::kSize;
    w.end = w.head + vocab;
    w.units = (w.end + Unit<BF16>::kElems - 1) / Unit<BF16>::kElems;
    return w;
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

// Unit u as floats; places outside the row hold -inf.
template <bool BF16>
__device__ __forceinline__ void load_unit(const Window &w, int u,
                                          float (&o)[Unit<BF16>::kElems]) {
    constexpr int E = Unit<BF16>::kElems;
    const int e0 = u * E;
    if (e0 >= w.head && e0 + E <= w.end) {
        const uint4 q = __ldcs(reinterpret_cast<const uint4 *>(w.base) + u);
        const uint32_t r[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (BF16) {
                o[2 * j] = bf16_lo(r[j]);
                o[2 * j + 1] = bf16_hi(r[j]);
            } else {
                o[j] = __uint_as_float(r[j]);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j)
            o[j] = e0 + j >= w.head && e0 + j < w.end ? load1<BF16>(w.base, e0 + j) : -INFINITY;
    }
}

// The unit of elements that is u in the source's window, into a row that may
// lie otherwise to the 16-byte boundaries (shift: destination head - source
// head).
template <bool BF16>
__device__ __forceinline__ void store_unit(const Window &src, const Window &dst, int u,
                                           const float (&v)[Unit<BF16>::kElems]) {
    constexpr int E = Unit<BF16>::kElems;
    const int e0 = u * E;
    if (src.head == dst.head && e0 >= src.head && e0 + E <= src.end) {
        uint4 q;
        if constexpr (BF16)
            q = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                           pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        else
            q = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                           __float_as_uint(v[3]));
        __stcs(reinterpret_cast<uint4 *>(dst.base) + u, q);
        return;
    }
    const int shift = dst.head - src.head;
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (e0 + j >= src.head && e0 + j < src.end) store1<BF16>(dst.base, e0 + j + shift, v[j]);
}

// Zeros in the units [u0, u1) of a row, by `threads` threads.
template <bool BF16>
__device__ __forceinline__ void zero_units(const Window &w, int first, int step) {
    constexpr int E = Unit<BF16>::kElems;
    float z[E];
#pragma unroll
    for (int j = 0; j < E; ++j) z[j] = 0.f;
    for (int u = first; u < w.units; u += step) store_unit<BF16>(w, w, u, z);
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

// exp((x - m) / tau).  The difference comes first: a product of the type's
// lowest value and the scale would leave the range.
__device__ __forceinline__ float exp_of(float x, float m, Scale s) {
    const float d = x - m;
    return exp2f(fmaf(d, s.hi, d * s.lo));
}

// (m, s) = the pair of both parts of a row: s counts exp((x - m) / tau).  An
// empty part has m = -inf and s = 0.
__device__ __forceinline__ float2 join(float2 a, float2 b, Scale scale) {
    const float m = fmaxf(a.x, b.x);
    const float base = m == -INFINITY ? 0.f : m;
    return make_float2(m, a.y * exp_of(a.x, base, scale) + b.y * exp_of(b.x, base, scale));
}

// Row kernel: cluster of C CTAs per row; thread t of CTA c holds the units
// (c * UPT + k) * THREADS + t, k < UPT.
template <bool BF16, int THREADS, int UPT, int MODE>
__global__ void __launch_bounds__(THREADS)
    row_kernel(const __grid_constant__ LogitsArgs a) {
    constexpr int E = Unit<BF16>::kElems;
    constexpr int WARPS = THREADS / 32;
    const Scale scale = {a.scale, a.scale_lo};
    __shared__ float2 s_warp[WARPS];
    __shared__ float2 s_cta[16];
    const cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t row = blockIdx.x / C;
    if (C > 1) cluster.barrier_arrive();  // every CTA runs before its memory is written

    const int64_t target = load_index(a.target, row, a.target_bytes);
    float weight = 1.f;
    if constexpr (MODE == kPolicy) weight = a.w[row];
    const bool live = target >= 0 && weight != 0.f;
    const Window g = a.g.data ? window_of<BF16>(a.g, row, a.vocab) : Window{};
    const bool first = rank == 0 && threadIdx.x == 0;
    if (!live) {
        if (C > 1) cluster.barrier_wait();
        if (MODE == kPolicy && a.g.data)
            zero_units<BF16>(g, rank * THREADS + threadIdx.x, C * THREADS);
        if (first) {
            a.logp[row] = 0.f;
            if constexpr (MODE == kPolicy)
                for (int j = 0; j < kTerms; ++j) a.terms[row * kTerms + j] = 0.f;
            if constexpr (MODE == kPref) a.coef[row] = 0.f;
        }
        return;
    }
    const Window x = window_of<BF16>(a.x, row, a.vocab);
    float v[UPT][E];
    const int u0 = rank * UPT * THREADS + threadIdx.x;
#pragma unroll
    for (int k = 0; k < UPT; ++k) {
        const int u = u0 + k * THREADS;
        if (u < x.units) {
            load_unit<BF16>(x, u, v[k]);
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) v[k][j] = -INFINITY;
        }
    }
    const float xt = target < a.vocab ? load1<BF16>(x.base, x.head + (int)target) : NAN;
    float old = 0.f, ref = 0.f, adv = 0.f;
    if constexpr (MODE == kPolicy) {
        old = a.old[row];
        adv = a.adv[row];
        if (a.ref) ref = a.ref[row];
    }

    float mt = -INFINITY;
#pragma unroll
    for (int k = 0; k < UPT; ++k)
#pragma unroll
        for (int j = 0; j < E; ++j) mt = fmaxf(mt, v[k][j]);
    const float base = mt == -INFINITY ? 0.f : mt;
    float st = 0.f;
#pragma unroll
    for (int k = 0; k < UPT; ++k)
#pragma unroll
        for (int j = 0; j < E; ++j) {
            v[k][j] = exp_of(v[k][j], base, scale);
            st += v[k][j];
        }

    // the row's maximum and sum, in an order that depends on the grid alone
    float2 q = make_float2(mt, st);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        float2 o;
        o.x = __shfl_xor_sync(0xffffffffu, q.x, off);
        o.y = __shfl_xor_sync(0xffffffffu, q.y, off);
        q = join(q, o, scale);
    }
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = q;
    __syncthreads();
    q = s_warp[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i) q = join(q, s_warp[i], scale);
    if (C > 1) {
        cluster.barrier_wait();
        if (threadIdx.x < C) *cluster.map_shared_rank(&s_cta[rank], threadIdx.x) = q;
        cluster.sync();
        q = s_cta[0];
        for (int i = 1; i < C; ++i) q = join(q, s_cta[i], scale);
    }
    const float m = q.x, z = q.y;
    // a row without a finite logit leaves z = 0: -inf - -inf
    const float logp = z > 0.f ? (xt - m) * a.inv_temp - logf(z) : NAN;

    if constexpr (MODE == kPolicy) {
        const float r = expf(logp - old);
        const float free = r * adv;
        const float bound = fminf(fmaxf(r, a.lo), a.hi) * adv;
        const bool act = free <= bound;
        const float d = ref - logp;
        const float back = a.kl != 0.f ? expf(d) : 1.f;
        if (first) {
            a.logp[row] = logp;
            float *t = a.terms + row * kTerms;
            t[0] = -weight * (act || free != free ? free : bound);
            t[1] = a.ref ? weight * (expf(d) - d - 1.f) : 0.f;
            t[2] = act ? 0.f : weight;
        }
        if (!a.g.data) return;
        const float k = weight * (a.kl * (1.f - back) - (act || free != free ? free : 0.f)) *
                        a.inv_temp;
        // this thread's values are exp((x - base) / tau), all 0 where it has no
        // finite logit
        const float f = -k * (z > 0.f ? (mt == -INFINITY ? 0.f : exp_of(base, m, scale) / z) : NAN);
        const int ut = (x.head + (int)target) / E;
#pragma unroll
        for (int i = 0; i < UPT; ++i) {
            const int u = u0 + i * THREADS;
            if (u >= x.units) break;
#pragma unroll
            for (int j = 0; j < E; ++j) v[i][j] *= f;
            if (u == ut) {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (ut * E + j == x.head + (int)target) v[i][j] += k;
            }
            store_unit<BF16>(x, g, u, v[i]);
        }
    } else if (first) {
        a.logp[row] = logp;
        if constexpr (MODE == kPref) {
            a.stats[row] = make_float2(m, z > 0.f ? 1.f / z : NAN);
            a.coef[row] = 0.f;
        }
    }
}

// Sum over the block in a fixed order (fp64); valid in every thread.
template <int THREADS>
__device__ __forceinline__ double block_total(double v, double *sh) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    for (int i = 0; i < THREADS / 32; ++i) s += sh[i];
    __syncthreads();
    return s;
}

__global__ void __launch_bounds__(1024) policy_terms_kernel(const __grid_constant__ LogitsArgs a) {
    __shared__ double sh[32];
    double s[kTerms] = {};
    for (int64_t r = threadIdx.x; r < a.n; r += 1024)
        for (int j = 0; j < kTerms; ++j) s[j] += (double)a.terms[r * kTerms + j];
    for (int j = 0; j < kTerms; ++j) s[j] = block_total<1024>(s[j], sh);
    if (threadIdx.x == 0) {
        a.terms_out[0] = (float)(s[0] + (double)a.kl * s[1]);
        for (int j = 0; j < kTerms; ++j) a.terms_out[1 + j] = (float)s[j];
    }
}

// Log ratios, losses and the rows' coefficients: one warp a pair, then one
// sum over the pairs.
__global__ void __launch_bounds__(1024) pairs_kernel(const __grid_constant__ LogitsArgs a) {
    __shared__ double sh[32];
    const int lane = threadIdx.x & 31;
    double sum = 0.0;
    for (int64_t k = threadIdx.x >> 5; k < a.pairs; k += 32) {
        int64_t lo[2], hi[2];
        double R[2];
        for (int i = 0; i < 2; ++i) {
            lo[i] = load_index(a.cu, 2 * k + i, a.cu_bytes);
            hi[i] = load_index(a.cu, 2 * k + i + 1, a.cu_bytes);
            lo[i] = lo[i] < 0 ? 0 : lo[i];
            hi[i] = hi[i] > a.n ? a.n : hi[i];
            double s = 0.0;
            for (int64_t r = lo[i] + lane; r < hi[i]; r += 32)
                if (load_index(a.target, r, a.target_bytes) >= 0)
                    s += (double)a.logp[r] - (a.ref ? (double)a.ref[r] : 0.0);
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
            R[i] = s;
        }
        const double z = a.beta * (R[0] - R[1]);
        const double t = exp(-fabs(z));
        // -log sigmoid(z) = log(1 + exp(-|z|)) + max(-z, 0)
        sum += log1p(t) + (z < 0.0 ? (1.0 - a.eps) * -z : a.eps * z);
        const double sig = z >= 0.0 ? 1.0 / (1.0 + t) : t / (1.0 + t);
        const double slope = (sig - (1.0 - a.eps)) * a.beta / (double)a.pairs;
        if (lane < 2) a.ratios[2 * k + lane] = (float)R[lane];
        if (a.g.data)
            for (int i = 0; i < 2; ++i)
                for (int64_t r = lo[i] + lane; r < hi[i]; r += 32)
                    if (load_index(a.target, r, a.target_bytes) >= 0)
                        a.coef[r] = (float)(i ? -slope : slope);
    }
    if (lane) sum = 0.0;
    sum = block_total<1024>(sum, sh);
    if (threadIdx.x == 0) a.loss[0] = a.pairs ? (float)(sum / (double)a.pairs) : 0.f;
}

// The preference loss's gradient: k ([j = a] - exp((x_j - m) / tau) / z).
template <bool BF16>
__global__ void __launch_bounds__(512) grad_kernel(const __grid_constant__ LogitsArgs a) {
    constexpr int E = Unit<BF16>::kElems;
    const int64_t row = blockIdx.x;
    const Window g = window_of<BF16>(a.g, row, a.vocab);
    const int64_t target = load_index(a.target, row, a.target_bytes);
    const float k = a.coef[row] * a.inv_temp;
    if (target < 0 || k == 0.f) {
        zero_units<BF16>(g, threadIdx.x, 512);
        return;
    }
    const Window x = window_of<BF16>(a.x, row, a.vocab);
    const float2 q = a.stats[row];
    const Scale scale = {a.scale, a.scale_lo};
    const float f = -k * q.y;
    const int at = target < a.vocab ? x.head + (int)target : -1;
    for (int u = threadIdx.x; u < x.units; u += 512) {
        float v[E];
        load_unit<BF16>(x, u, v);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            v[j] = exp_of(v[j], q.x, scale) * f;
            if (u * E + j == at) v[j] += k;
        }
        store_unit<BF16>(x, g, u, v);
    }
}

// Launch a row kernel: THREADS * UPT units a CTA, as many CTAs as the row's
// window takes, and more where there are too few rows for the SMs.
template <bool BF16, int THREADS, int EPT, int MODE>
cudaError_t launch_rows_as(const LogitsArgs &a, int sm_count, cudaStream_t stream) {
    constexpr int E = Unit<BF16>::kElems, UPT = EPT / E;
    const int units = (a.vocab + 2 * (E - 1)) / E;
    int C = (units + THREADS * UPT - 1) / (THREADS * UPT);
    if (C > 8) return cudaErrorInvalidValue;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)C;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.n * C));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, row_kernel<BF16, THREADS, UPT, MODE>, a);
}

template <bool BF16, int MODE>
cudaError_t launch_rows(const LogitsArgs &a, int sm_count, cudaStream_t stream) {
    if (a.n == 0) return cudaSuccess;
    if (a.vocab <= 4096 - 8) return launch_rows_as<BF16, 128, 32, MODE>(a, sm_count, stream);
    if (a.vocab <= 131072 - 8) return launch_rows_as<BF16, 512, 32, MODE>(a, sm_count, stream);
    return launch_rows_as<BF16, 512, 72, MODE>(a, sm_count, stream);
}

}  // namespace

cudaError_t launch_token_logprobs(const LogitsArgs &a, aloco_dtype dtype, int sm_count,
                                  cudaStream_t stream) {
    return dtype == ALOCO_BF16 ? launch_rows<true, kFwd>(a, sm_count, stream)
                               : launch_rows<false, kFwd>(a, sm_count, stream);
}

cudaError_t launch_policy_loss(const LogitsArgs &a, aloco_dtype dtype, int sm_count,
                               cudaStream_t stream) {
    const cudaError_t e = dtype == ALOCO_BF16 ? launch_rows<true, kPolicy>(a, sm_count, stream)
                                              : launch_rows<false, kPolicy>(a, sm_count, stream);
    if (e != cudaSuccess) return e;
    policy_terms_kernel<<<1, 1024, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_preference_loss(const LogitsArgs &a, aloco_dtype dtype, int sm_count,
                                   cudaStream_t stream) {
    const cudaError_t e = dtype == ALOCO_BF16 ? launch_rows<true, kPref>(a, sm_count, stream)
                                              : launch_rows<false, kPref>(a, sm_count, stream);
    if (e != cudaSuccess) return e;
    pairs_kernel<<<1, 1024, 0, stream>>>(a);
    if (a.g.data && a.n) {
        if (dtype == ALOCO_BF16)
            grad_kernel<true><<<(unsigned)a.n, 512, 0, stream>>>(a);
        else
            grad_kernel<false><<<(unsigned)a.n, 512, 0, stream>>>(a);
    }
    return cudaGetLastError();
}

}  // namespace aloco
