// Global norm of many gradient tensors, and clipping by it.
//
//   norm = sqrt(sum_i sum_j g_ij^2),   c = min(1, max_norm / (norm + 1e-6)),
//   g' = c g
//
// The tensors are cut into stretches of equal length, listed in device
// memory; blocks take stretches in turn, so that a set of many small and few
// large tensors spreads evenly.  Both kernels stream, bound by HBM from some 1e7
// elements on: the norm reads every gradient once (137.8e6 fp32 in 83.9 us, 0.97
// of the copy rate), the scaling reads it again, what L2 has kept of it from
// there, and writes it (1.1e9 bf16 into a bf16 vector in 961 us with the norm;
// two reads and a write take 973 at the copy rate).
#include <algorithm>

#include "aloco_grads.h"
#include "aloco_sync_kernel.cuh"
#include "aloco_units.cuh"

namespace aloco {

namespace {

constexpr int kUnits = 4;  // 16-byte units a thread has in flight

template <bool BF16>
__device__ __forceinline__ float grad1(const void *p, int64_t e) {
    if constexpr (BF16)
        return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[e] << 16);
    else
        return reinterpret_cast<const float *>(p)[e];
}
template <bool BF16>
__device__ __forceinline__ void put1(void *p, int64_t e, float v) {
    if constexpr (BF16)
        reinterpret_cast<__nv_bfloat16 *>(p)[e] = __float2bfloat16_rn(v);
    else
        reinterpret_cast<float *>(p)[e] = v;
}

template <bool BF16>
__device__ __forceinline__ void widen(const uint4 &q, float (&o)[BF16 ? 8 : 4]) {
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
}

// Elements before p's next 16-byte boundary, at most n.
template <bool BF16>
__device__ __forceinline__ int head_of(const void *p, int n) {
    const int h = (int)((16 - ((uintptr_t)p & 15)) & 15) / (BF16 ? 2 : 4);
    return h < n ? h : n;
}

// A sum of squares: in fp32 with what its additions rounded away (fp64 units are
// rare here: with fp64 sums the norm of 3e6 elements took 14 us, most of it in
// the reduction), and in fp64 what fp32 cannot hold.
struct Squares {
    float s = 0.f, rest = 0.f;
    double wide = 0.0;
    __device__ __forceinline__ void add(float x) {
        const float t = s + x, b = t - s;
        rest += (s - (t - b)) + (x - b);
        s = t;
    }
    // x: a sum of at most 32 squares.  Below 1e25 the fp32 sum of 2^44 of them
    // stays in range, and above 1e-30 squares that round away do not matter.
    __device__ __forceinline__ static bool fits(float x) { return x >= 1e-30f && x <= 1e25f; }
};

// Add the squares of up to 32 elements that this thread holds as units.
template <bool BF16>
__device__ __forceinline__ void add_squares(Squares &acc, const uint4 (&q)[kUnits]) {
    constexpr int E = BF16 ? 8 : 4;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        float v[E];
        widen<BF16>(q[k], v);
#pragma unroll
        for (int j = 0; j < E; ++j) s = fmaf(v[j], v[j], s);
    }
    if (Squares::fits(s)) {
        acc.add(s);
        return;
    }
    for (int k = 0; k < kUnits; ++k) {
        const uint32_t any = (q[k].x | q[k].y | q[k].z | q[k].w) &
                             (BF16 ? 0x7fff7fffu : 0x7fffffffu);
        if (!any) continue;
        float v[E];
        widen<BF16>(q[k], v);
        for (int j = 0; j < E; ++j) acc.wide += (double)v[j] * (double)v[j];
    }
}

template <bool BF16>
__device__ __forceinline__ void add_chunk(Squares &acc, const void *p, int n) {
    const int h = head_of<BF16>(p, n);
    constexpr int E = BF16 ? 8 : 4;
    const int units = (n - h) / E;
    const uint4 *u = reinterpret_cast<const uint4 *>(static_cast<const char *>(p) +
                                                     (size_t)h * (BF16 ? 2 : 4));
    for (int i = threadIdx.x; i < units; i += kUnits * kGradBlock) {
        uint4 q[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int j = i + k * kGradBlock;
            q[k] = j < units ? __ldg(u + j) : make_uint4(0, 0, 0, 0);
        }
        add_squares<BF16>(acc, q);
    }
    const int tail = h + units * E;
    for (int e = threadIdx.x; e < h + n - tail; e += kGradBlock) {
        const float x = grad1<BF16>(p, e < h ? e : tail + e - h);
        if (Squares::fits(x * x))
            acc.add(x * x);
        else
            acc.wide += (double)x * (double)x;
    }
}

// The block's sum in a fixed order, in thread 0.  fp64 only where some thread
// has a part of its own there.
__device__ __forceinline__ Squares block_sum(Squares v) {
    __shared__ float2 sh[kGradBlock / 32];
    __shared__ double sh_wide[kGradBlock / 32];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const float s = __shfl_down_sync(0xffffffffu, v.s, off);
        const float r = __shfl_down_sync(0xffffffffu, v.rest, off);
        v.add(s);
        v.rest += r;
    }
    const bool wide = __syncthreads_or(v.wide != 0.0);  // (NaN is not 0)
    if (wide)
        for (int off = 16; off > 0; off >>= 1)
            v.wide += __shfl_down_sync(0xffffffffu, v.wide, off);
    if ((threadIdx.x & 31) == 0) {
        sh[threadIdx.x >> 5] = make_float2(v.s, v.rest);
        sh_wide[threadIdx.x >> 5] = v.wide;
    }
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < kGradBlock / 32; ++w) {
            v.add(sh[w].x);
            v.rest += sh[w].y;
            if (wide) v.wide += sh_wide[w];
        }
    return v;
}

__global__ void __launch_bounds__(kGradBlock) grad_norm_kernel(const __grid_constant__ GradArgs a) {
    Squares acc;
    for (int c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
        const GradChunk k = a.chunks[c];
        if (k.bf16)
            add_chunk<true>(acc, k.p, k.n);
        else
            add_chunk<false>(acc, k.p, k.n);
    }
    acc = block_sum(acc);
    __shared__ bool last;
    if (threadIdx.x == 0) {
        a.partials[blockIdx.x] = {acc.s, acc.rest, acc.wide};
        __threadfence();
        last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    acc = Squares();
    for (int b = threadIdx.x; b < (int)gridDim.x; b += kGradBlock) {
        const float4 p = __ldcg(reinterpret_cast<const float4 *>(a.partials + b));
        acc.add(p.x);
        acc.rest += p.y;
        const double w = __hiloint2double(__float_as_int(p.w), __float_as_int(p.z));
        if (w != 0.0) acc.wide += w;
    }
    acc = block_sum(acc);
    if (threadIdx.x == 0) {
        const float norm = acc.wide == 0.0 ? sqrtf(acc.s + acc.rest)
                                           : (float)sqrt((double)acc.s + (double)acc.rest + acc.wide);
        a.norm[0] = norm;
        // (a norm beyond fp32 is inf, whose factor is 0)
        const float c = a.max_norm / (norm + 1e-6f);
        *a.factor = c > 1.f ? 1.f : c;
        *a.ticket = 0;
    }
}

// E elements, scaled and rounded, as 16 or 32 bytes (OBF16: 8 or 16) at o.
template <bool OBF16, int E>
__device__ __forceinline__ void put_unit(char *o, const float (&v)[E]) {
    if constexpr (OBF16) {
        uint32_t r[E / 2];
#pragma unroll
        for (int e = 0; e < E / 2; ++e) r[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
        if constexpr (E == 8)
            __stcs(reinterpret_cast<uint4 *>(o), make_uint4(r[0], r[1], r[2], r[3]));
        else
            __stcs(reinterpret_cast<uint2 *>(o), make_uint2(r[0], r[1]));
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 4)
            __stcs(reinterpret_cast<float4 *>(o) + e / 4,
                   make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]));
    }
}

// N units of the source, kGradBlock apart, scaled into o.
template <bool BF16, bool OBF16, int N>
__device__ __forceinline__ void scale_units(const uint4 *u, char *o, float c) {
    constexpr int E = BF16 ? 8 : 4, OB = E * (OBF16 ? 2 : 4);
    uint4 q[N];
#pragma unroll
    for (int k = 0; k < N; ++k) q[k] = __ldcs(u + k * kGradBlock);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float v[E];
        widen<BF16>(q[k], v);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= c;
        put_unit<OBF16>(o + k * kGradBlock * OB, v);
    }
}

// N 16-byte units of the destination, kGradBlock apart, from elements at src.
template <bool BF16, bool OBF16, int N>
__device__ __forceinline__ void gather_units(const char *src, char *o, float c) {
    constexpr int E = OBF16 ? 8 : 4, IS = BF16 ? 2 : 4;
    float v[N][E];
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) v[k][e] = grad1<BF16>(src + k * kGradBlock * E * IS, e);
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[k][e] *= c;
        put_unit<OBF16>(o + k * kGradBlock * 16, v[k]);
    }
}

// N 16-byte units of the destination, kGradBlock apart, each from two
// neighbouring ones of a source of the same type.
template <bool BF16, int N>
__device__ __forceinline__ void join_and_scale(const uint4 *u, char *o, int bytes, float c) {
    constexpr int E = BF16 ? 8 : 4;
    uint4 q[N], r[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        q[k] = __ldg(u + k * kGradBlock);
        r[k] = __ldg(u + k * kGradBlock + 1);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float v[E];
        widen<BF16>(join_units(q[k], r[k], bytes), v);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= c;
        put_unit<BF16>(o + k * kGradBlock * 16, v);
    }
}

// c g of one stretch, rounded once to the destination's type, in 16-byte units
// of the source where those lie on a boundary of the destination too.  Else (a
// tensor's place in the flat vector is the sum of the sizes before it) units
// are the destination's: made of two neighbouring ones where both have one type
// (5e8 bf16 at odd places: 481 against 554 us element by element), and of the
// source's elements one by one where not; neighbours share their lines in L1,
// while stores of single elements would each go to L2.
template <bool BF16, bool OBF16>
__device__ __forceinline__ void scale_chunk(const void *p, void *out, int n, float c) {
    constexpr int IS = BF16 ? 2 : 4, OS = OBF16 ? 2 : 4, OB = 16 / IS * OS;
    const char *src = static_cast<const char *>(p);
    char *dst = static_cast<char *>(out);
    int h = head_of<BF16>(p, n), end;
    if (((uintptr_t)(dst + h * OS) & ((OB < 16 ? OB : 16) - 1)) == 0) {
        const int units = (n - h) / (16 / IS);
        const uint4 *u = reinterpret_cast<const uint4 *>(src + h * IS);
        char *o = dst + h * OS;
        int i = threadIdx.x;
        for (; i + (kUnits - 1) * kGradBlock < units; i += kUnits * kGradBlock)
            scale_units<BF16, OBF16, kUnits>(u + i, o + (size_t)i * OB, c);
        for (; i < units; i += kGradBlock)
            scale_units<BF16, OBF16, 1>(u + i, o + (size_t)i * OB, c);
        end = h + units * (16 / IS);
    } else if constexpr (BF16 == OBF16) {
        constexpr int E = 16 / IS;
        const int us = (n - h) / E;           // whole units of the source, from element h
        const int hd = head_of<OBF16>(out, n);
        // unit j of the destination, from element hd, begins in unit j - lower of
        // the source, (hd - h) mod E elements on
        const int lower = hd < h, on = hd - h + lower * E;
        const int units = max(0, min((n - hd) / E - lower, us - 1));
        const uint4 *u = reinterpret_cast<const uint4 *>(src + h * IS);
        h = hd + lower * E;
        char *o = dst + h * OS;
        int i = threadIdx.x;
        for (; i + kGradBlock < units; i += 2 * kGradBlock)
            join_and_scale<BF16, 2>(u + i, o + (size_t)i * 16, 16 - on * IS, c);
        for (; i < units; i += kGradBlock)
            join_and_scale<BF16, 1>(u + i, o + (size_t)i * 16, 16 - on * IS, c);
        end = h + units * E;
    } else {
        h = head_of<OBF16>(out, n);
        const int units = (n - h) / (16 / OS);
        src += h * IS;
        char *o = dst + h * OS;
        int i = threadIdx.x;
        for (; i + kGradBlock < units; i += 2 * kGradBlock)
            gather_units<BF16, OBF16, 2>(src + (size_t)i * (16 / OS) * IS, o + (size_t)i * 16, c);
        for (; i < units; i += kGradBlock)
            gather_units<BF16, OBF16, 1>(src + (size_t)i * (16 / OS) * IS, o + (size_t)i * 16, c);
        end = h + units * (16 / OS);
    }
    for (int e = threadIdx.x; e < h + n - end; e += kGradBlock) {
        const int at = e < h ? e : end + e - h;
        put1<OBF16>(out, at, c * grad1<BF16>(p, at));
    }
}

// OUT: 0 in place, 1 into an fp32 vector, 2 into a bf16 one.
template <int OUT>
__global__ void __launch_bounds__(kGradBlock, 4)
    grad_scale_kernel(const __grid_constant__ GradArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");  // for the norm
    const float c = __ldcg(a.factor);
    if (OUT == 0 && c == 1.f) return;
    for (int i = blockIdx.x; i < a.n_chunks; i += gridDim.x) {
        const GradChunk k = a.chunks[a.n_chunks - 1 - i];  // the end first: L2 still has it
        void *o = OUT == 0 ? k.p : static_cast<char *>(a.out) + (size_t)k.at * (OUT == 2 ? 2 : 4);
        if (k.bf16)
            scale_chunk<true, OUT != 1>(k.p, o, k.n, c);
        else
            scale_chunk<false, OUT == 2>(k.p, o, k.n, c);
    }
}

}  // namespace

int grad_norm_blocks(int sm_count, int n_chunks) {
    const int most = sm_count * 4;  // as many as are resident at once
    return n_chunks < 1 ? 1 : n_chunks < most ? n_chunks : most;
}

cudaError_t launch_grad_norm(const GradArgs &a, int sm_count, cudaStream_t stream) {
    grad_norm_kernel<<<grad_norm_blocks(sm_count, a.n_chunks), kGradBlock, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_grad_scale(const GradArgs &a, int sm_count, cudaStream_t stream) {
    if (a.n_chunks == 0) return cudaSuccess;
    cudaLaunchAttribute attr = {};  // its blocks come while the norm's last ones end
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min(a.n_chunks, sm_count * 32));
    cfg.blockDim = dim3(kGradBlock);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, !a.out ? grad_scale_kernel<0>
                                    : a.out_bf16 ? grad_scale_kernel<2> : grad_scale_kernel<1>, a);
}

}  // namespace aloco
