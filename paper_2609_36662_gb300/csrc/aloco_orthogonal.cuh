// What the kernels of the orthogonalised updates share: where matrices come from
// and go to.
#pragma once

#include <cuda_bf16.h>

#include "aloco_orthogonal.h"

namespace aloco {
namespace {

// The group whose numbers start at or before `t`.
template <typename F>
__device__ __forceinline__ int find_group(const OrthoArgs &a, int t, F first) {
    int g = 0;
    while (g + 1 < a.n_groups && first(a.g[g + 1]) <= t) ++g;
    return g;
}

struct Place {
    int worker;
    int64_t at;
};
__device__ __forceinline__ Place find_place(const OrthoArgs &a, const OrthoGroup &g, int matrix) {
    const int i = g.skip + matrix, w = i / g.period;
    return {w, a.place[g.first + (i - w * g.period)]};
}

__device__ __forceinline__ uint32_t pack(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack(uint32_t u) {
    return __half22float2(*reinterpret_cast<const __half2 *>(&u));
}

__device__ __forceinline__ float param_load(const void *p, int64_t i, int bf16) {
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i])
                : static_cast<const float *>(p)[i];
}
__device__ __forceinline__ void param_store(void *p, int64_t i, int bf16, float v) {
    if (bf16)
        static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
    else
        static_cast<float *>(p)[i] = v;
}

// U = g + mu b' (or b') with b' = mu b + g.
struct Momentum {
    float mu;
    int nesterov;
    __device__ __forceinline__ float next(float b, float g) const { return fmaf(mu, b, g); }
    __device__ __forceinline__ float u(float b1, float g) const {
        return nesterov ? fmaf(mu, b1, g) : b1;
    }
};

// Four values from element i on, in one access (i and p suit it).
__device__ __forceinline__ float4 load4(const void *p, int64_t i, int bf16) {
    if (!bf16) return *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i);
    const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(p) + i);
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u),
                       __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
}

// A matrix as the caller has it.
struct Source {
    const void *in;
    float *momentum;                 // null: U is what lies there
    int64_t at, stride;              // element (0, 0); to the next row
    int bf16;
    bool by4;                        // four values of a row at once
    Momentum mo;

    __device__ __forceinline__ Source(const OrthoArgs &a, const OrthoGroup &g, int matrix) {
        const Place p = find_place(a, g, matrix);
        const bool muon = a.source == kSourceMuon;
        in = a.in[muon ? p.worker : 0];
        momentum = muon ? a.momentum[p.worker] : nullptr;
        at = muon ? p.at : p.at * a.batch_stride;
        stride = muon ? g.cols : a.row_stride;
        bf16 = a.in_bf16;
        mo = {a.mu, a.nesterov};
        const uintptr_t first = (uintptr_t)in + at * (bf16 ? 2 : 4);
        by4 = !((g.cols | stride) & 3) && !(first & (bf16 ? 7 : 15)) &&
              !(momentum && ((uintptr_t)(momentum + at) & 15));
    }
    __device__ __forceinline__ float u(int64_t e) const {
        const float g = param_load(in, at + e, bf16);
        return momentum ? mo.u(mo.next(momentum[at + e], g), g) : g;
    }
    __device__ __forceinline__ float4 u4(int64_t e) const {
        float4 g = load4(in, at + e, bf16);
        if (momentum) {
            const float4 b = load4(momentum, at + e, 0);
            g.x = mo.u(mo.next(b.x, g.x), g.x);
            g.y = mo.u(mo.next(b.y, g.y), g.y);
            g.z = mo.u(mo.next(b.z, g.z), g.z);
            g.w = mo.u(mo.next(b.w, g.w), g.w);
        }
        return g;
    }
};

// The sum of 16 squares in fp32; of values whose squares leave its range in fp64.
__device__ __forceinline__ double squares(const float (&v)[16]) {
    float s = 0.f, top = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        s = fmaf(v[j], v[j], s);
        top = fmaxf(top, fabsf(v[j]));
    }
    if (top < 1e18f && (top > 1e-12f || top == 0.f) && s == s) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int j = 0; j < 16; ++j) d += (double)v[j] * (double)v[j];
    return d;
}

// Where a matrix's result goes: parameters p <- p decay + step o, or o itself.
struct Result {
    void *p;
    int64_t at, stride;              // element (0, 0); to the next row in memory
    int bf16, update, tall;          // tall: a row in memory is a column of X
    bool whole;                      // 16-byte pieces of rows are aligned
    float decay, step;

    __device__ __forceinline__ Result(const OrthoArgs &a, const OrthoGroup &g, int group,
                                      int matrix) {
        const Place place = find_place(a, g, matrix);
        update = a.source == kSourceMuon;
        p = a.out[update ? place.worker : 0];
        at = update ? place.at : place.at * g.rows * g.cols;
        stride = g.cols;
        bf16 = a.out_bf16;
        tall = g.tall;
        decay = a.decay;
        step = a.step[group];
        whole = !((uintptr_t)address(0) & 15) && !(stride & (bf16 ? 7 : 3));
    }
    __device__ __forceinline__ char *address(int64_t e) const {
        return static_cast<char *>(p) + (at + e) * (bf16 ? 2 : 4);
    }
    __device__ __forceinline__ float value(float x, float o) const {
        return update ? fmaf(x, decay, step * o) : o;
    }
};

}  // namespace
}  // namespace aloco
