// Orthogonal factors by Newton-Schulz products on the tensor cores: X <- (a +
// b A + c A A) X with A = X X^T, some steps of it, for many matrices at once.
#include <cuda_bf16.h>

#include "aloco_orthogonal.h"
#include "aloco_tc.cuh"

namespace aloco {
namespace {

constexpr int kThreads = 256;
constexpr int kHalfTile = 128;       // a CTA's rows of a tile
constexpr int kK = 64;               // k-elements of a slot: 128 bytes a row
constexpr int kBox = 64;             // rows of a copied box
constexpr int kBoxBytes = kBox * kK * 2;
constexpr int kSlotBytes = 4 * kBoxBytes;  // two boxes of either operand
constexpr int kSlots = 6;
constexpr int kSharedBytes = kSlots * kSlotBytes + 1024 + 256;
constexpr int kEpilogueWarp = 4;     // the first of four

struct Tile {
    int group, matrix, row, col;     // row, col: in tiles
};

// The group whose numbers start at or before `t`.
template <typename F>
__device__ __forceinline__ int find_group(const OrthoArgs &a, int t, F first) {
    int g = 0;
    while (g + 1 < a.n_groups && first(a.g[g + 1]) <= t) ++g;
    return g;
}

template <int kWhat>
__device__ __forceinline__ Tile find_tile(const OrthoArgs &a, int t, int tile) {
    Tile f;
    if constexpr (kWhat == kUpdate) {
        f.group = find_group(a, t, [](const OrthoGroup &g) { return g.up0; });
        const OrthoGroup &g = a.g[f.group];
        t -= g.up0;
        f.matrix = t / g.up_tiles;
        t -= f.matrix * g.up_tiles;
        const int rows = (g.m + tile - 1) / tile;
        f.col = t / rows;            // the rows of P first: X's columns stay in L2
        f.row = t - f.col * rows;
    } else {
        f.group = find_group(a, t, [](const OrthoGroup &g) { return g.sym0; });
        const OrthoGroup &g = a.g[f.group];
        t -= g.sym0;
        f.matrix = t / g.sym_tiles;
        t -= f.matrix * g.sym_tiles;
        // row r of the lower triangle holds tiles r (r + 1) / 2 ..
        int r = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while (r * (r + 1) / 2 > t) --r;
        while ((r + 1) * (r + 2) / 2 <= t) ++r;
        f.row = r;
        f.col = t - r * (r + 1) / 2;
    }
    return f;
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

// 32 columns of row r of a symmetric matrix: those at or left of the diagonal as
// they lie, and mirrored.
//   v: the values; on the diagonal what goes beside the matrix has been taken
//   out (they are 0 there).
__device__ __forceinline__ void store_symmetric(__half *o, int m, int ld, int r, int c0,
                                                bool crossing, int lane, const float (&v)[32]) {
    if (!crossing) {                 // all c < r
        if (r < m) {
            __half *row = o + (int64_t)r * ld + c0;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                reinterpret_cast<uint4 *>(row)[q] =
                    make_uint4(pack(v[8 * q], v[8 * q + 1]), pack(v[8 * q + 2], v[8 * q + 3]),
                               pack(v[8 * q + 4], v[8 * q + 5]), pack(v[8 * q + 6], v[8 * q + 7]));
        }
        // two lanes join their values of two columns: rows behind the last are
        // padding up to a multiple of 8 and hold whatever comes
        const bool even = !(lane & 1);
        __half *col = o + (int64_t)(c0 + (lane & 1)) * ld + (r & ~1);
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const uint32_t own = pack(v[2 * q], v[2 * q + 1]);
            const uint32_t other = __shfl_xor_sync(~0u, own, 1);
            const uint32_t both = __byte_perm(own, other, even ? 0x5410 : 0x3276);
            if (r < ld) *reinterpret_cast<uint32_t *>(col + (int64_t)2 * q * ld) = both;
        }
        return;
    }
    if (r >= m) return;
#pragma unroll
    for (int q = 0; q < 32; ++q) {
        const int c = c0 + q;
        if (c > r) continue;
        const __half h = __float2half_rn(v[q]);
        o[(int64_t)r * ld + c] = h;
        if (c < r) o[(int64_t)c * ld + r] = h;
    }
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

// One product of all matrices.  Persistent CTAs (pairs) take tiles in turn: one
// thread copies operands into a ring of slots, one issues the products into one
// of two accumulators, four warps write the other one's tile.  A wait that runs
// out leaves NaN in the tile, and with it in the matrix.
//   kGram    A = X X^T, lower tiles, mirrored; the diagonal in fp32
//   kPoly    P = b A + c A A, the same
//   kUpdate  X <- a X + P X, or the result
// A and P are symmetric: half their tiles are computed.
template <int kWhat, int kCtas>
__global__ void __launch_bounds__(kThreads, 1)
    ortho_product_kernel(const __grid_constant__ OrthoArgs args) {
    constexpr int kTile = kHalfTile * kCtas;
    constexpr uint32_t kDesc = product_desc(kTile, kTile, kWhat == kUpdate);
    extern __shared__ char raw[];
    const uint32_t smem = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t bars = smem + kSlots * kSlotBytes;
    const auto full = [&](int s) { return bars + 8 * s; };
    const auto empty = [&](int s) { return bars + 8 * (kSlots + s); };
    const auto acc_full = [&](int s) { return bars + 8 * (2 * kSlots + s); };
    const auto acc_empty = [&](int s) { return bars + 8 * (2 * kSlots + 2 + s); };
    const uint32_t drained = bars + 8 * (2 * kSlots + 4);
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = kCtas == 1 ? 0 : cluster_rank();
    const int first = blockIdx.x / kCtas, stride = gridDim.x / kCtas;
    const int tiles = kWhat == kUpdate ? args.up_tiles : args.sym_tiles;

    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(acc_full(s), 1);
            mbar_init(acc_empty(s), 4 * kCtas);
        }
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_alloc<kCtas>(smem_addr(&s_tmem), 2 * kTile);
    tc_fence_before();
    __syncthreads();
    if constexpr (kCtas == 2) cluster_sync();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    grid_go();
    grid_wait();

    const auto depth = [&](const OrthoGroup &g) { return kWhat == kGram ? g.n : g.m; };

    if (warp == 0 && lane == 0) {
        // operands were written by ordinary stores of the kernel before
        asm volatile("fence.proxy.async;" ::: "memory");
        int slot = 0, issued = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int t = first; t < tiles && ok; t += stride) {
            const Tile f = find_tile<kWhat>(args, t, kTile);
            const int chunks = (depth(args.g[f.group]) + kK - 1) / kK;
            const CUtensorMap *ma = &args.map_a[f.group], *mb = &args.map_b[f.group];
            const int ra = f.row * kTile + (int)rank * kHalfTile;
            const int rb = f.col * kTile + (int)rank * kHalfTile;
            for (int k = 0; k < chunks; ++k) {
                if (!(ok = mbar_wait(empty(slot), phase ^ 1, &s_abort))) break;
                const uint32_t bar = kCtas == 1 ? full(slot) : cluster_addr(full(slot), 0);
                const uint32_t at = smem + slot * kSlotBytes;
                if (rank == 0) mbar_arrive_expect_tx(full(slot), kCtas * kSlotBytes);
                const bool skip = args.test_stall1 && blockIdx.x == 0 &&
                                  issued == args.test_stall1 - 1;
                if (!skip) {
                    tensor_load<kCtas>(at, ma, k * kK, ra, f.matrix, bar);
                    tensor_load<kCtas>(at + kBoxBytes, ma, k * kK, ra + kBox, f.matrix, bar);
                    if constexpr (kWhat == kUpdate) {
                        tensor_load<kCtas>(at + 2 * kBoxBytes, mb, rb, k * kK, f.matrix, bar);
                        tensor_load<kCtas>(at + 3 * kBoxBytes, mb, rb + kBox, k * kK, f.matrix,
                                           bar);
                    } else {
                        tensor_load<kCtas>(at + 2 * kBoxBytes, mb, k * kK, rb, f.matrix, bar);
                        tensor_load<kCtas>(at + 3 * kBoxBytes, mb, k * kK, rb + kBox, f.matrix,
                                           bar);
                    }
                }
                ++issued;
                if (++slot == kSlots) slot = 0, phase ^= 1;
            }
        }
        if (!ok) {
            s_abort = 1;
            // copies in flight land before the block ends (each slot's last use)
            if (rank == 0)
                for (int i = issued > kSlots ? issued - kSlots : 0; i < issued; ++i)
                    mbar_wait(full(i % kSlots), (i / kSlots) & 1, nullptr);
        }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        int slot = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        bool ok = true;
        for (int t = first; t < tiles && ok; t += stride) {
            const Tile f = find_tile<kWhat>(args, t, kTile);
            const int K = depth(args.g[f.group]);
            if (!(ok = mbar_wait(acc_empty(acc), acc_phase ^ 1, &s_abort))) break;
            tc_fence_after();
            for (int k = 0; k < K; k += kK) {
                if (!(ok = mbar_wait(full(slot), phase, &s_abort))) break;
                tc_fence_after();
                const uint32_t a0 = smem + slot * kSlotBytes, b0 = a0 + 2 * kBoxBytes;
                // (what lies behind K is zeros)
                const int steps = min(kK, K - k + 15) / 16;
                for (int i = 0; i < steps; ++i) {
                    const uint64_t da = operand_desc(a0 + 32 * i, 16);
                    const uint64_t db = kWhat == kUpdate ? operand_desc(b0 + 2048 * i, kBoxBytes)
                                                         : operand_desc(b0 + 32 * i, 16);
                    product<kCtas>(tmem + acc * kTile, da, db, kDesc, (k | i) != 0);
                }
                product_commit<kCtas>(empty(slot));
                if (++slot == kSlots) slot = 0, phase ^= 1;
            }
            if (!ok) break;
            product_commit<kCtas>(acc_full(acc));
            if (acc) acc_phase ^= 1;
            acc ^= 1;
        }
        if (!ok) {
            s_abort = 1;
            // products in flight end before their accumulators are given back
            product_commit<kCtas>(drained);
            mbar_wait(drained, 0, nullptr);
        }
    } else if (warp >= kEpilogueWarp) {
        const int quad = warp - kEpilogueWarp;
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int t = first; t < tiles; t += stride) {
            const Tile f = find_tile<kWhat>(args, t, kTile);
            const OrthoGroup &g = args.g[f.group];
            const bool ok = mbar_wait(acc_full(acc), acc_phase, &s_abort);
            if (!ok) s_abort = 1;
            tc_fence_after();
            const int m = g.m, r0 = f.row * kTile + (int)rank * kHalfTile + quad * 32;
            const int r = r0 + lane, limit = kWhat == kUpdate ? g.n : m;
            const Place place = kWhat == kUpdate && args.last ? find_place(args, g, f.matrix)
                                                              : Place{0, 0};
#pragma unroll 1
            for (int q = 0; q < kTile / 32; ++q) {
                const int c0 = f.col * kTile + q * 32;
                if (r0 >= m || c0 >= limit) break;
                if (kWhat != kUpdate && c0 > r0 + 31) break;
                uint32_t u[32];
                tmem_read32(tmem + acc * kTile + q * 32 + (quad << 21), u);
                tmem_ready();
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    v[i] = ok ? __uint_as_float(u[i]) : __int_as_float(0x7fffffff);
                if constexpr (kWhat == kGram) {
                    const bool crossing = c0 + 31 >= r0;
                    float *diag = g.diag + (int64_t)f.matrix * m;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        v[i] *= 1.f / (kOrthoScale * kOrthoScale);
                        if (c0 + i == r) {
                            if (r < m) diag[r] = v[i];
                            v[i] = 0.f;
                        }
                    }
                    store_symmetric(g.a + (int64_t)f.matrix * m * g.lda, m, g.lda, r, c0, crossing,
                                    lane, v);
                } else if constexpr (kWhat == kPoly) {
                    const bool crossing = c0 + 31 >= r0;
                    const float *diag = g.diag + (int64_t)f.matrix * m;
                    const float dr = r < m ? diag[r] : 0.f;
                    const uint4 *row = reinterpret_cast<const uint4 *>(
                        g.a + ((int64_t)f.matrix * m + min(r, m - 1)) * g.lda + c0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint4 w = c0 + 8 * i < m ? row[i] : make_uint4(0, 0, 0, 0);
                        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int c = c0 + 8 * i + j;
                            const float2 h = unpack(ws[j / 2]);
                            const float a = j & 1 ? h.y : h.x;
                            const float dc = c < m ? diag[c] : 0.f;
                            float &x = v[8 * i + j];
                            if (c == r) {
                                if (r < m)
                                    g.lead[(int64_t)f.matrix * m + r] =
                                        args.ca + args.cb * dr + args.cc * (dr * dr + x);
                                x = 0.f;
                            } else {
                                x = args.cb * a + args.cc * ((dr + dc) * a + x);
                            }
                        }
                    }
                    store_symmetric(g.p + (int64_t)f.matrix * m * g.lda, m, g.lda, r, c0, crossing,
                                    lane, v);
                } else {
                    if (r >= m) continue;
                    const int64_t base = args.source == kSourceMatrix
                                             ? place.at * g.rows * g.cols
                                             : place.at;
                    const float lead = g.lead[(int64_t)f.matrix * m + r];
                    const int64_t at = ((int64_t)f.matrix * m + r) * g.ldx + c0;
                    const uint4 *hi = reinterpret_cast<const uint4 *>(g.x[args.next ^ 1] + at);
                    uint4 *lo = reinterpret_cast<uint4 *>(g.lo + at);
                    uint4 *to = reinterpret_cast<uint4 *>(g.x[args.next] + at);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (c0 + 8 * i >= g.n) continue;
                        const uint4 h4 = hi[i], l4 = lo[i];
                        const uint32_t hs[4] = {h4.x, h4.y, h4.z, h4.w};
                        const uint32_t ls[4] = {l4.x, l4.y, l4.z, l4.w};
                        uint32_t nh[4], nl[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 h = unpack(hs[j]), l = unpack(ls[j]);
                            float &x = v[8 * i + 2 * j], &y = v[8 * i + 2 * j + 1];
                            x = fmaf(lead, h.x + l.x, x);
                            y = fmaf(lead, h.y + l.y, y);
                            nh[j] = pack(x, y);
                            const float2 b = unpack(nh[j]);
                            nl[j] = pack(x - b.x, y - b.y);
                        }
                        if (!args.last) {
                            to[i] = make_uint4(nh[0], nh[1], nh[2], nh[3]);
                            lo[i] = make_uint4(nl[0], nl[1], nl[2], nl[3]);
                            continue;
                        }
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int c = c0 + 8 * i + j;
                            if (c >= g.n) break;
                            const int64_t e = base + (g.tall ? (int64_t)c * g.cols + r
                                                                 : (int64_t)r * g.cols + c);
                            const float o = v[8 * i + j] * (1.f / kOrthoScale);
                            if (args.source == kSourceMatrix) {
                                param_store(args.out[0], e, 1, o);
                            } else {
                                void *p = args.out[place.worker];
                                const float x = param_load(p, e, args.out_bf16);
                                param_store(p, e, args.out_bf16,
                                            fmaf(x, args.decay, args.step[f.group] * o));
                            }
                        }
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (kCtas == 1)
                    mbar_arrive(acc_empty(acc));
                else
                    mbar_arrive_cluster(cluster_addr(acc_empty(acc), 0));
            }
            if (acc) acc_phase ^= 1;
            acc ^= 1;
        }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (kCtas == 2) cluster_sync();
    tc_fence_after();
    if (warp == 2) tmem_free<kCtas>(tmem, 2 * kTile);
}

// ------------------------------------------------- from the caller's matrices

__device__ __forceinline__ float in_load(const void *p, int64_t i, int bf16) {
    return param_load(p, i, bf16);
}

// u = g + mu b' (or b') with b' = mu b + g.
struct Momentum {
    float mu;
    int nesterov;
    __device__ __forceinline__ float next(float b, float g) const { return fmaf(mu, b, g); }
    __device__ __forceinline__ float u(float b1, float g) const {
        return nesterov ? fmaf(mu, b1, g) : b1;
    }
};

__device__ __forceinline__ float load_u(const OrthoArgs &a, const OrthoGroup &g, const Place &p,
                                        int64_t i) {
    if (a.source == kSourceMatrix) {
        const int64_t r = i / g.cols;
        return in_load(a.in[0], p.at * a.batch_stride + r * a.row_stride + (i - r * g.cols),
                       a.in_bf16);
    }
    const Momentum mo{a.mu, a.nesterov};
    const float gr = in_load(a.in[p.worker], p.at + i, a.in_bf16);
    return mo.u(mo.next(a.momentum[p.worker][p.at + i], gr), gr);
}

__device__ __forceinline__ double block_sum(double s, double *shared) {
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = s;
    __syncthreads();
    s = 0.0;
    for (int i = 0; i < (int)blockDim.x / 32; ++i) s += shared[i];
    __syncthreads();
    return s;
}

// Sums of squares of the matrices' stretches: fp32 over 16 values, fp64 beyond;
// what leaves fp32's range is squared in fp64.
__global__ void __launch_bounds__(kThreads) ortho_norm_kernel(const __grid_constant__ OrthoArgs args) {
    __shared__ double shared[kThreads / 32];
    grid_go();
    grid_wait();
    const int gi = find_group(args, blockIdx.x, [](const OrthoGroup &g) { return g.norm0; });
    const OrthoGroup &g = args.g[gi];
    const int b = blockIdx.x - g.norm0, matrix = b / g.chunks, chunk = b - matrix * g.chunks;
    const Place place = find_place(args, g, matrix);
    const int64_t total = (int64_t)g.rows * g.cols;
    const int64_t begin = (int64_t)chunk * g.chunk, end = min(total, begin + g.chunk);
    double sum = 0.0;
    for (int64_t i = begin + threadIdx.x; i < end; i += 16 * kThreads) {
        float v[16], s = 0.f, top = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int64_t e = i + j * kThreads;
            v[j] = e < end ? load_u(args, g, place, e) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            s = fmaf(v[j], v[j], s);
            top = fmaxf(top, fabsf(v[j]));
        }
        if (top < 1e18f && (top > 1e-12f || top == 0.f) && s == s) {
            sum += (double)s;
        } else {
#pragma unroll 1
            for (int j = 0; j < 16; ++j) sum += (double)v[j] * (double)v[j];
        }
    }
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) g.partial[(int64_t)matrix * g.chunks + chunk] = sum;
}

constexpr int kPrep = 64;            // rows and columns of a prepared tile

// X = u 2^8 / (|u| + eps) as a pair of fp16, transposed where the matrix is
// tall, and the new momentum.
__global__ void __launch_bounds__(kThreads) ortho_prepare_kernel(const __grid_constant__ OrthoArgs args) {
    __shared__ double shared[kThreads / 32];
    __shared__ float tile[kPrep][kPrep + 1];
    grid_go();
    grid_wait();
    const int gi = find_group(args, blockIdx.x, [](const OrthoGroup &g) { return g.prep0; });
    const OrthoGroup &g = args.g[gi];
    const int across = (g.cols + kPrep - 1) / kPrep, down = (g.rows + kPrep - 1) / kPrep;
    int b = blockIdx.x - g.prep0;
    const int matrix = b / (across * down);
    b -= matrix * across * down;
    const int r0 = b / across * kPrep, c0 = b % across * kPrep;
    const Place place = find_place(args, g, matrix);

    double s = 0.0;
    for (int i = threadIdx.x; i < g.chunks; i += kThreads)
        s += g.partial[(int64_t)matrix * g.chunks + i];
    s = block_sum(s, shared);
    const double factor = (double)kOrthoScale / (sqrt(s) + args.eps);
    const bool plain = factor > 1e-30 && factor < 1e30;
    const float f = (float)factor;

    const Momentum mo{args.mu, args.nesterov};
    for (int i = threadIdx.x; i < kPrep * kPrep; i += kThreads) {
        const int y = i / kPrep, x = i % kPrep, r = r0 + y, c = c0 + x;
        float u = 0.f;
        if (r < g.rows && c < g.cols) {
            if (args.source == kSourceMatrix) {
                u = in_load(args.in[0],
                            place.at * args.batch_stride + r * args.row_stride + c,
                            args.in_bf16);
            } else {
                const int64_t e = place.at + (int64_t)r * g.cols + c;
                const float gr = in_load(args.in[place.worker], e, args.in_bf16);
                float *buf = args.momentum[place.worker] + e;
                const float b1 = mo.next(*buf, gr);
                *buf = b1;
                u = mo.u(b1, gr);
            }
        }
        tile[y][x] = plain ? u * f : (float)((double)u * factor);
    }
    __syncthreads();
    const int64_t base = (int64_t)matrix * g.m * g.ldx;
    for (int i = threadIdx.x; i < kPrep * kPrep; i += kThreads) {
        const int y = i / kPrep, x = i % kPrep;
        const int r = (g.tall ? c0 : r0) + y, c = (g.tall ? r0 : c0) + x;
        if (r >= g.m || c >= g.n) continue;
        const float v = g.tall ? tile[x][y] : tile[y][x];
        const __half h = __float2half_rn(v);
        g.x[0][base + (int64_t)r * g.ldx + c] = h;
        g.lo[base + (int64_t)r * g.ldx + c] = __float2half_rn(v - __half2float(h));
    }
}

template <typename K>
cudaError_t launch(K kernel, const OrthoArgs &a, int grid, int ctas, int smem,
                   cudaStream_t stream) {
    if (grid == 0) return cudaSuccess;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(grid);
    c.blockDim = dim3(kThreads);
    c.dynamicSmemBytes = smem;
    c.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {(unsigned)ctas, 1, 1};
    c.attrs = at;
    c.numAttrs = ctas > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&c, kernel, a);
}

template <int kWhat, int kCtas>
cudaError_t launch_product(const OrthoArgs &a, int sm_count, cudaStream_t stream) {
    static PerDevice ready;
    const auto kernel = ortho_product_kernel<kWhat, kCtas>;
    const int d = PerDevice::device();
    if (!ready.get(d)) {
        const cudaError_t e = cudaFuncSetAttribute(
            kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes);
        if (e != cudaSuccess) return e;
        ready.set(d, 1);
    }
    const int tiles = kWhat == kUpdate ? a.up_tiles : a.sym_tiles;
    const int most = sm_count / kCtas;
    return launch(kernel, a, (tiles < most ? tiles : most) * kCtas, kCtas, kSharedBytes, stream);
}

}  // namespace

int ortho_pair_tile() { return 2 * kHalfTile; }

cudaError_t launch_ortho_norm(const OrthoArgs &a, cudaStream_t stream) {
    return launch(ortho_norm_kernel, a, a.norm_blocks, 1, 0, stream);
}

cudaError_t launch_ortho_prepare(const OrthoArgs &a, cudaStream_t stream) {
    return launch(ortho_prepare_kernel, a, a.prep_blocks, 1, 0, stream);
}

cudaError_t launch_ortho_product(OrthoProduct what, const OrthoArgs &a, int ctas, int sm_count,
                                 cudaStream_t stream) {
    if (ctas == 1)
        return what == kGram   ? launch_product<kGram, 1>(a, sm_count, stream)
               : what == kPoly ? launch_product<kPoly, 1>(a, sm_count, stream)
                               : launch_product<kUpdate, 1>(a, sm_count, stream);
    return what == kGram   ? launch_product<kGram, 2>(a, sm_count, stream)
           : what == kPoly ? launch_product<kPoly, 2>(a, sm_count, stream)
                           : launch_product<kUpdate, 2>(a, sm_count, stream);
}

}  // namespace aloco
