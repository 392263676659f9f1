// Global norm of many gradient tensors, and clipping by it.
//
//   norm = sqrt(sum_i sum_j g_ij^2),   c = min(1, max_norm / (norm + 1e-6)),
//   g' = c g
//
// The tensors are cut into stretches of equal length, listed in device
// memory; blocks take stretches in turn, so that a set of many small and few
// large tensors spreads evenly.  Both kernels stream: the norm reads every
// gradient once, the scaling reads it again and writes it.
#include "aloco_grads.h"
#include "aloco_sync_kernel.cuh"

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

// Sum of the squares of up to 32 elements that this thread holds as units.
// In fp32; where that leaves its range (a square above 3.4e38, or all so
// small that theirs round away), again in fp64.
template <bool BF16>
__device__ __forceinline__ double squares(const uint4 (&q)[kUnits]) {
    constexpr int E = BF16 ? 8 : 4;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        float v[E];
        widen<BF16>(q[k], v);
#pragma unroll
        for (int j = 0; j < E; ++j) s = fmaf(v[j], v[j], s);
    }
    if (s >= 1e-30f && s <= FLT_MAX) return (double)s;
    double d = 0.0;
    for (int k = 0; k < kUnits; ++k) {
        const uint32_t any = (q[k].x | q[k].y | q[k].z | q[k].w) &
                             (BF16 ? 0x7fff7fffu : 0x7fffffffu);
        if (!any) continue;
        float v[E];
        widen<BF16>(q[k], v);
        for (int j = 0; j < E; ++j) d += (double)v[j] * (double)v[j];
    }
    return d;
}

template <bool BF16>
__device__ __forceinline__ double chunk_squares(const void *p, int n) {
    double acc = 0.0;
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
        acc += squares<BF16>(q);
    }
    const int tail = h + units * E;
    for (int e = threadIdx.x; e < h + n - tail; e += kGradBlock) {
        const double x = (double)grad1<BF16>(p, e < h ? e : tail + e - h);
        acc += x * x;
    }
    return acc;
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double sh[kGradBlock / 32];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_down_sync(0xffffffffu, v, off);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kGradBlock / 32; ++w) s += sh[w];
    return s;
}

__global__ void __launch_bounds__(kGradBlock) grad_norm_kernel(const __grid_constant__ GradArgs a) {
    double acc = 0.0;
    for (int c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
        const GradChunk k = a.chunks[c];
        acc += k.bf16 ? chunk_squares<true>(k.p, k.n) : chunk_squares<false>(k.p, k.n);
    }
    double s = block_sum(acc);
    __shared__ bool last;
    if (threadIdx.x == 0) {
        a.partials[blockIdx.x] = s;
        __threadfence();
        last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    s = 0.0;
    for (int b = threadIdx.x; b < (int)gridDim.x; b += kGradBlock) s += __ldcg(a.partials + b);
    __syncthreads();
    s = block_sum(s);
    if (threadIdx.x == 0) {
        const double norm = sqrt(s);
        a.norm[0] = (float)norm;
        double c = a.max_norm / (norm + 1e-6);
        if (c > 1.0) c = 1.0;
        *a.factor = c;
        *a.ticket = 0;
    }
}

// c g of one stretch, rounded once to the destination's type.
template <bool BF16, bool OBF16>
__device__ __forceinline__ void scale_chunk(const void *p, void *out, int n, float c) {
    constexpr int E = BF16 ? 8 : 4;
    const int h = head_of<BF16>(p, n);
    const int units = (n - h) / E;
    const uint4 *u = reinterpret_cast<const uint4 *>(static_cast<const char *>(p) +
                                                     (size_t)h * (BF16 ? 2 : 4));
    constexpr int OB = E * (OBF16 ? 2 : 4);  // bytes of a unit's elements in out
    char *o = static_cast<char *>(out) + (size_t)h * (OBF16 ? 2 : 4);
    const bool whole = ((uintptr_t)o & ((OB < 16 ? OB : 16) - 1)) == 0;
    for (int i = threadIdx.x; i < units; i += kUnits * kGradBlock) {
        uint4 q[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int j = i + k * kGradBlock;
            if (j < units) q[k] = __ldcs(u + j);
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int j = i + k * kGradBlock;
            if (j >= units) break;
            float v[E];
            widen<BF16>(q[k], v);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] *= c;
            if (!whole) {
#pragma unroll
                for (int e = 0; e < E; ++e) put1<OBF16>(o, (int64_t)j * E + e, v[e]);
            } else if constexpr (OBF16) {
                uint32_t r[E / 2];
#pragma unroll
                for (int e = 0; e < E / 2; ++e) r[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
                if constexpr (BF16)
                    __stcs(reinterpret_cast<uint4 *>(o) + j, make_uint4(r[0], r[1], r[2], r[3]));
                else
                    __stcs(reinterpret_cast<uint2 *>(o) + j, make_uint2(r[0], r[1]));
            } else {
#pragma unroll
                for (int e = 0; e < E; e += 4)
                    __stcs(reinterpret_cast<float4 *>(o) + (int64_t)j * (E / 4) + e / 4,
                           make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]));
            }
        }
    }
    const int tail = h + units * E;
    for (int e = threadIdx.x; e < h + n - tail; e += kGradBlock) {
        const int at = e < h ? e : tail + e - h;
        put1<OBF16>(out, at, c * grad1<BF16>(p, at));
    }
}

__global__ void __launch_bounds__(kGradBlock) grad_scale_kernel(const __grid_constant__ GradArgs a) {
    const double cd = __ldcg(a.factor);
    if (!a.out && cd == 1.0) return;
    const float c = (float)cd;
    for (int i = blockIdx.x; i < a.n_chunks; i += gridDim.x) {
        const GradChunk k = a.chunks[a.n_chunks - 1 - i];  // the end first: L2 still has it
        if (!a.out) {
            if (k.bf16)
                scale_chunk<true, true>(k.p, k.p, k.n, c);
            else
                scale_chunk<false, false>(k.p, k.p, k.n, c);
            continue;
        }
        char *o = static_cast<char *>(a.out) + (size_t)k.at * (a.out_bf16 ? 2 : 4);
        if (k.bf16) {
            if (a.out_bf16)
                scale_chunk<true, true>(k.p, o, k.n, c);
            else
                scale_chunk<true, false>(k.p, o, k.n, c);
        } else {
            if (a.out_bf16)
                scale_chunk<false, true>(k.p, o, k.n, c);
            else
                scale_chunk<false, false>(k.p, o, k.n, c);
        }
    }
}

}  // namespace

int grad_norm_blocks(int sm_count, int n_chunks) {
    const int most = sm_count * 8;
    return n_chunks < 1 ? 1 : n_chunks < most ? n_chunks : most;
}

cudaError_t launch_grad_norm(const GradArgs &a, int sm_count, cudaStream_t stream) {
    grad_norm_kernel<<<grad_norm_blocks(sm_count, a.n_chunks), kGradBlock, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_grad_scale(const GradArgs &a, int sm_count, cudaStream_t stream) {
    if (a.n_chunks == 0) return cudaSuccess;
    grad_scale_kernel<<<grad_norm_blocks(sm_count, a.n_chunks), kGradBlock, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace aloco
