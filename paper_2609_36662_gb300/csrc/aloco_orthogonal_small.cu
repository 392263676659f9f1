// Orthogonal factors of matrices whose smaller side is at most 128, all steps in
// one kernel: a matrix stays in the registers and shared memory of a CTA, or of a
// cluster whose CTAs take its columns.
#include "aloco_orthogonal.cuh"
#include "aloco_tc.cuh"

namespace aloco {
namespace {

constexpr int kThreads = 256;        // eight warps: a quarter of the rows, half of the columns
constexpr int kRows = kOrthoSmallSide;
constexpr int kCols = kOrthoSmallCols;       // of a CTA
constexpr int kBlock = kRows * 128;  // 64 columns of 128 rows in fp16, 128 bytes swizzled
constexpr int kXBytes = kCols / 64 * kBlock, kABytes = kRows / 64 * kBlock;
constexpr int kShareBytes = kRows * kRows * 4;  // a CTA's part of A
constexpr int kSharedBytes = kXBytes + 2 * kABytes + kShareBytes + 1024;
constexpr int kEach = kCols / 2;     // columns of a thread
constexpr uint32_t kTmemColumns = 512;  // 128 of A and P, 256 of X

// The 16-byte piece that holds columns c .. c + 7 (c a multiple of 8) of row r.
__device__ __forceinline__ uint32_t piece_at(int r, int c) {
    return (uint32_t)(c / 64 * kBlock + r * 128 + ((c % 64 / 8) ^ (r & 7)) * 16);
}
__device__ __forceinline__ void store_shared(uint32_t at, const uint4 &q) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(q.x), "r"(q.y), "r"(q.z),
                 "r"(q.w)
                 : "memory");
}
__device__ __forceinline__ uint4 load_shared(uint32_t at) {
    uint4 q;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
                 : "r"(at)
                 : "memory");
    return q;
}
__device__ __forceinline__ float4 load_peer(uint32_t at) {
    float4 q;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w)
                 : "r"(at)
                 : "memory");
    return q;
}
__device__ __forceinline__ void store_peer(uint32_t at, const uint4 &q) {
    asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(q.x), "r"(q.y),
                 "r"(q.z), "r"(q.w)
                 : "memory");
}

// A 16-byte piece of a part of A in fp32: four columns of row r, turned so that a
// warp's rows spread over the banks.
__device__ __forceinline__ uint32_t share_at(int r, int c) {
    return (uint32_t)(r * kRows * 4 + ((c / 4) ^ (r & 7)) * 16);
}
// The same of this CTA's X, which lies where A, P and the parts come to lie.
__device__ __forceinline__ uint32_t stage_at(int r, int c) {
    return (uint32_t)(r * kCols * 4 + ((c / 4) ^ (r & 7)) * 16 + c % 4 * 4);
}
static_assert(2 * kABytes + kShareBytes >= kRows * kCols * 4, "X's stage");

// This CTA's part of a matrix in the order of memory: `runs` stretches of `length`
// elements, taken `each` (1 or 4) at a time.
struct Walk {
    int per, units;
    float inverse;
    __device__ __forceinline__ Walk(int runs, int length, int each)
        : per(length / each), units(runs * per), inverse(1.f / (float)max(1, per)) {}
    // (units < 2^15: the quotient is at least 1 / 512 away from a whole number)
    __device__ __forceinline__ int run(int unit) const {
        return (int)(((float)unit + 0.5f) * inverse);
    }
};

// Matrices of the groups whose clusters have this launch's size.  Thread (row,
// half): columns half * 128 .. + 127 of its CTA's 256, of X in fp32 in registers;
// its fp16 values, A and P lie in shared memory as operands, K-major and MN-major
// in one.  Parts of A are added over the cluster in rank order.  A CTA whose wait
// runs out goes on with NaN, which its cluster gets with its part of A.
//
// A step is a chain of latencies (three products, their fences and reads, and the
// cluster's exchange: about 4 us, 6 with it), where the products' kernel takes 20: one
// 2048 x 16 matrix takes 33 us in all and 4 workers' two of 512 x 64 take 47, 122 and
// 101 there.  64 of 16 x 2048, by clusters of 8, take 157 us in four rounds.
__global__ void __launch_bounds__(kThreads, 1)
    ortho_small_kernel(const __grid_constant__ OrthoArgs args) {
    extern __shared__ char raw[];
    __shared__ uint32_t s_tmem;
    __shared__ float s_diag[kRows], s_lead[kRows];
    __shared__ double s_sum[kThreads / 32];
    __shared__ double s_total;       // the CTA's squares, for its cluster
    __shared__ float s_factor;       // where fp32 does for it
    __shared__ uint64_t s_bar;
    const uint32_t smem = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t xs = smem, as = xs + kXBytes, ps = as + kABytes, share = ps + kABytes;
    const uint32_t bar = smem_addr(&s_bar);
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int quad = warp % 4, half = warp / 4, r = quad * 32 + lane;

    const int ctas = args.small_ctas, rank = ctas > 1 ? (int)cluster_rank() : 0;
    const int at = blockIdx.x / ctas;
    const int gi = find_group(args, at, [](const OrthoGroup &g) { return g.small0; });
    const OrthoGroup &g = args.g[gi];
    const int matrix = at - g.small0, m = g.m;
    // this CTA's columns of X
    const int each = ((g.n + ctas - 1) / ctas + 15) & ~15;
    const int first = min(g.n, rank * each), cols = min(g.n - first, each);

    if (tid == 0) {
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc<1>(smem_addr(&s_tmem), kTmemColumns);
    for (uint32_t i = tid * 16; i < kXBytes; i += kThreads * 16)
        store_shared(smem + i, make_uint4(0, 0, 0, 0));
    grid_go();
    grid_wait();

    // U, its norm, and the new momentum, as they lie in memory; through shared
    // memory to the threads' rows
    const Source s(args, g, matrix);
    const Result to(args, g, gi, matrix);
    const int runs = g.tall ? cols : m, length = g.tall ? m : cols;
    const int64_t origin = g.tall ? (int64_t)first * s.stride : first;
    // (squares in fp32, where they fit: the SM adds two doubles a clock)
    float near = 0.f;
    double far = 0.0;
    const auto take = [&](const float *v, int n) {
        float sq = 0.f, top = 0.f;
        for (int j = 0; j < n; ++j) {
            sq = fmaf(v[j], v[j], sq);
            top = fmaxf(top, fabsf(v[j]));
        }
        if (top < 1e16f && (top > 1e-14f || top == 0.f) && sq == sq) {
            near += sq;
        } else {
            for (int j = 0; j < n; ++j) far += (double)v[j] * (double)v[j];
        }
    };
    const auto stage = [&](int run, int l) {   // element l of a run
        return as + (g.tall ? stage_at(l, run) : stage_at(run, l));
    };
    if (s.by4) {
        const Walk w(runs, length, 4);
        for (int i = tid; i < w.units; i += 8 * kThreads) {
            float4 q[8], o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int u = i + k * kThreads, run = w.run(u);
                if (u >= w.units) continue;
                const int64_t e = s.at + origin + run * s.stride + (u - run * w.per) * 4;
                q[k] = load4(s.in, e, s.bf16);
                if (s.momentum) o[k] = load4(s.momentum, e, 0);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int u = i + k * kThreads, run = w.run(u), l = (u - run * w.per) * 4;
                if (u >= w.units) continue;
                float *v = &q[k].x, *b = &o[k].x;
                if (s.momentum) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        b[j] = s.mo.next(b[j], v[j]);
                        v[j] = s.mo.u(b[j], v[j]);
                    }
                    *reinterpret_cast<float4 *>(s.momentum + s.at + origin + run * s.stride + l) =
                        o[k];
                    if (u % 8 == 0) fetch_l2(to.address(origin + run * s.stride + l));
                }
                take(v, 4);
                if (!g.tall) {
                    store_shared(as + stage_at(run, l),
                                 make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]),
                                            __float_as_uint(v[2]), __float_as_uint(v[3])));
                    continue;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(stage(run, l + j)), "f"(v[j])
                                 : "memory");
            }
        }
    } else {
        const Walk w(runs, length, 1);
        for (int i = tid; i < w.units; i += 16 * kThreads) {
            float v[16], b[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int u = i + k * kThreads, run = w.run(u);
                if (u >= w.units) continue;
                const int64_t e = s.at + origin + run * s.stride + (u - run * w.per);
                v[k] = param_load(s.in, e, s.bf16);
                if (s.momentum) b[k] = s.momentum[e];
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int u = i + k * kThreads, run = w.run(u), l = u - run * w.per;
                if (u >= w.units) continue;
                if (s.momentum) {
                    const float next = s.mo.next(b[k], v[k]);
                    s.momentum[s.at + origin + run * s.stride + l] = next;
                    v[k] = s.mo.u(next, v[k]);
                    if (lane == 0) fetch_l2(to.address(origin + run * s.stride + l));
                }
                take(&v[k], 1);
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(stage(run, l)), "f"(v[k]) : "memory");
            }
        }
    }
    double sum = (double)near + far;
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
    if (lane == 0) s_sum[warp] = sum;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    if (tid == 0) {
        double t = 0.0;
        for (int i = 0; i < kThreads / 32; ++i) t += s_sum[i];
        s_total = t;
    }
    if (ctas > 1)
        cluster_sync();
    else
        __syncthreads();
    if (tid == 0) {
        double total = s_total;
        if (ctas > 1) {
            total = 0.0;
            for (int p = 0; p < ctas; ++p) {
                double t;
                asm volatile("ld.shared::cluster.f64 %0, [%1];"
                             : "=d"(t)
                             : "r"(cluster_addr(smem_addr(&s_total), p))
                             : "memory");
                total += t;
            }
        }
        const bool usual = total > 1e-30 && total < 1e30 && args.eps < 1e30;
        s_factor = usual ? kOrthoScale / (sqrtf((float)total) + (float)args.eps) : 0.f;
        if (!usual) s_sum[0] = (double)kOrthoScale / (sqrt(total) + args.eps);
    }
    __syncthreads();
    const int j0 = half * kEach;
    const int count = r < m ? max(0, min(kEach, cols - j0)) : 0;  // of this thread
    float x[kEach];
#pragma unroll
    for (int j = 0; j < kEach; j += 4) {
        uint4 q = make_uint4(0, 0, 0, 0);
        if (j < count) q = load_shared(as + stage_at(r, j0 + j));
        x[j] = __uint_as_float(q.x);
        x[j + 1] = j + 1 < count ? __uint_as_float(q.y) : 0.f;
        x[j + 2] = j + 2 < count ? __uint_as_float(q.z) : 0.f;
        x[j + 3] = j + 3 < count ? __uint_as_float(q.w) : 0.f;
    }
    if (s_factor > 0.f) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) x[j] *= s_factor;
    } else {
        const double factor = s_sum[0];
#pragma unroll
        for (int j = 0; j < kEach; ++j) x[j] = (float)((double)x[j] * factor);
    }
    // (rows and columns of A and P that there are not)
    __syncthreads();
    for (uint32_t i = tid * 16; i < 2 * kABytes; i += kThreads * 16)
        store_shared(as + i, make_uint4(0, 0, 0, 0));

    // X's fp16 values: rows and columns that there are
    const auto show = [&] {
        if (r >= m) return;
#pragma unroll
        for (int j = 0; j < kEach; j += 8)
            if (j < count)
                store_shared(xs + piece_at(r, j0 + j),
                             make_uint4(pack(x[j], x[j + 1]), pack(x[j + 2], x[j + 3]),
                                        pack(x[j + 4], x[j + 5]), pack(x[j + 6], x[j + 7])));
    };
    show();

    const int wide = (m + 15) & ~15;                  // columns of A, k of P X
    const int deep = ctas > 1 ? (each + 15) & ~15 : (cols + 15) & ~15;
    const int a_end = min(wide, (half + 1) * 64);     // this thread's columns of A
    bool ok = true, stall = args.test_stall1 && blockIdx.x == 0;
    uint32_t phase = 0;
    // what all threads have written is seen by the products of thread 0, whose
    // end all wait for
    const auto products = [&](auto issue) {
        fence_proxy_async_smem();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (tid == 0 && ok && !stall) {
            issue();
            product_commit<1>(bar);
        }
        if (ok) ok = mbar_wait(bar, phase, nullptr);
        ok = __syncthreads_and(ok);
        if (ok) phase ^= 1;
        stall = false;
        tc_fence_after();
    };

#pragma unroll 1
    for (int step = 0; step < args.steps; ++step) {
        const float ca = args.coef[step][0], cb = args.coef[step][1], cc = args.coef[step][2];
        // A = X X^T of these columns
        products([&] {
            const uint32_t desc = product_desc(kRows, wide);
            for (int k = 0; k < deep; k += 16) {
                const uint64_t d = operand_desc(xs + k / 64 * kBlock + k % 64 * 2, 16);
                product<1>(tmem, d, d, desc, k != 0);
            }
        });
        for (int c = half * 64; c < a_end; c += 32) {
            uint32_t u[32];
            __syncwarp();
            tmem_read32(tmem + c + (quad << 21), u);
            if (r >= m) continue;
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i)
                v[i] = ok ? __uint_as_float(u[i]) * (1.f / (kOrthoScale * kOrthoScale)) : NAN;
            if (ctas > 1) {
#pragma unroll
                for (int i = 0; i < 32; i += 4)
                    store_shared(share + share_at(r, c + i),
                                 make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]),
                                            __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])));
                continue;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (c + i == r) {
                    s_diag[r] = v[i];
                    v[i] = 0.f;
                }
#pragma unroll
            for (int i = 0; i < 32; i += 8)
                if (c + i < wide)
                    store_shared(as + piece_at(r, c + i),
                                 make_uint4(pack(v[i], v[i + 1]), pack(v[i + 2], v[i + 3]),
                                            pack(v[i + 4], v[i + 5]), pack(v[i + 6], v[i + 7])));
        }
        if (ctas > 1) {
            cluster_sync();
            // rows of this rank: added, and written to every CTA
            const int rows = (m + ctas - 1) / ctas, pieces = wide / 8;
            const int begin = min(m, rank * rows), end = min(m, begin + rows);
            for (int i = tid; i < (end - begin) * pieces; i += kThreads) {
                const int row = begin + i / pieces, c = i % pieces * 8;
                float v[8] = {};
                for (int p = 0; p < ctas; ++p) {
                    const uint32_t base = cluster_addr(share, p);
                    const float4 lo = load_peer(base + share_at(row, c));
                    const float4 hi = load_peer(base + share_at(row, c + 4));
                    v[0] += lo.x, v[1] += lo.y, v[2] += lo.z, v[3] += lo.w;
                    v[4] += hi.x, v[5] += hi.y, v[6] += hi.z, v[7] += hi.w;
                }
                float own = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k == row) own = v[k], v[k] = 0.f;
                const uint4 q = make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]),
                                           pack(v[6], v[7]));
                for (int p = 0; p < ctas; ++p) {
                    store_peer(cluster_addr(as, p) + piece_at(row, c), q);
                    if (row >= c && row < c + 8)
                        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(
                                         cluster_addr(smem_addr(&s_diag[row]), p)),
                                     "f"(own)
                                     : "memory");
                }
            }
            asm volatile("fence.proxy.async;" ::: "memory");
            cluster_sync();
        }
        // P = b A + c A A
        products([&] {
            const uint32_t desc = product_desc(kRows, wide);
            for (int k = 0; k < wide; k += 16) {
                const uint64_t d = operand_desc(as + k / 64 * kBlock + k % 64 * 2, 16);
                product<1>(tmem, d, d, desc, k != 0);
            }
        });
        for (int c = half * 64; c < a_end; c += 32) {
            uint32_t u[32];
            __syncwarp();
            tmem_read32(tmem + c + (quad << 21), u);
            if (r >= m) continue;
            const float dr = s_diag[r], by_row = fmaf(cc, dr, cb);
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
                if (c + i >= wide) break;
                const uint4 w = load_shared(as + piece_at(r, c + i));
                const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int col = c + i + k;
                    const float2 h = unpack(ws[k / 2]);
                    const float dc = col < m ? s_diag[col] : 0.f, q = __uint_as_float(u[i + k]);
                    v[k] = fmaf(k & 1 ? h.y : h.x, fmaf(cc, dc, by_row), cc * q);
                    if (col == r) {
                        s_lead[r] = ca + cb * dr + cc * (dr * dr + q);
                        v[k] = 0.f;
                    }
                }
                store_shared(ps + piece_at(r, c + i),
                             make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]),
                                        pack(v[6], v[7])));
            }
        }
        // X <- a X + P X: rows of P by columns of X, which lie MN-major
        products([&] {
            const int n = min(kCols, deep);
            const uint32_t desc = product_desc(kRows, n) | kBMnMajor;
            for (int k = 0; k < wide; k += 16) {
                const uint64_t a = operand_desc(ps + k / 64 * kBlock + k % 64 * 2, 16);
                const uint64_t b = operand_desc(xs + k * 128, kBlock);
                product<1>(tmem + kRows, a, b, desc, k != 0);
            }
        });
        const float lead = r < m ? s_lead[r] : 0.f;
#pragma unroll
        for (int j = 0; j < kEach; j += 32) {
            if (j0 + j >= deep) break;               // (of the whole warp)
            uint32_t u[32];
            __syncwarp();
            tmem_read32(tmem + kRows + j0 + j + (quad << 21), u);
#pragma unroll
            for (int i = 0; i < 32; ++i) x[j + i] = fmaf(lead, x[j + i], __uint_as_float(u[i]));
        }
        if (step + 1 < args.steps) show();
    }
    if (!ok) {
        // products in flight end before their accumulators are given back
        if (tid == 0) {
            product_commit<1>(bar);
            mbar_wait(bar, phase, nullptr);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) x[j] = __int_as_float(0x7fffffff);
    }

    // the result, back the same way (peers have read their parts of A)
#pragma unroll
    for (int j = 0; j < kEach; j += 4)
        if (j < count)
            store_shared(as + stage_at(r, j0 + j),
                         make_uint4(__float_as_uint(x[j] * (1.f / kOrthoScale)),
                                    __float_as_uint(x[j + 1] * (1.f / kOrthoScale)),
                                    __float_as_uint(x[j + 2] * (1.f / kOrthoScale)),
                                    __float_as_uint(x[j + 3] * (1.f / kOrthoScale))));
    __syncthreads();
    const int64_t base = g.tall ? (int64_t)first * to.stride : first;
    const auto staged = [&](int run, int l) {
        float v;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(stage(run, l)) : "memory");
        return v;
    };
    if (to.whole) {
        const Walk w(runs, length, 4);
        for (int i = tid; i < w.units; i += 8 * kThreads) {
            float4 old[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int u = i + k * kThreads, run = w.run(u);
                if (u < w.units && to.update)
                    old[k] = load4(to.p, to.at + base + run * to.stride + (u - run * w.per) * 4,
                                   to.bf16);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int u = i + k * kThreads, run = w.run(u), l = (u - run * w.per) * 4;
                if (u >= w.units) continue;
                const float *o = &old[k].x;
                float v[4];
                if (!g.tall) {
                    const uint4 q = load_shared(as + stage_at(run, l));
                    v[0] = __uint_as_float(q.x);
                    v[1] = __uint_as_float(q.y);
                    v[2] = __uint_as_float(q.z);
                    v[3] = __uint_as_float(q.w);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = staged(run, l + j);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = to.value(o[j], v[j]);
                char *p = to.address(base + run * to.stride + l);
                if (to.bf16) {
                    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]),
                                         c = __floats2bfloat162_rn(v[2], v[3]);
                    *reinterpret_cast<uint2 *>(p) =
                        make_uint2(*reinterpret_cast<const uint32_t *>(&a),
                                   *reinterpret_cast<const uint32_t *>(&c));
                } else {
                    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
                }
            }
        }
    } else {
        const Walk w(runs, length, 1);
        for (int i = tid; i < w.units; i += 16 * kThreads) {
            float old[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int u = i + k * kThreads, run = w.run(u);
                if (u < w.units && to.update)
                    old[k] = param_load(to.address(base + run * to.stride + (u - run * w.per)), 0,
                                        to.bf16);
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int u = i + k * kThreads, run = w.run(u), l = u - run * w.per;
                if (u < w.units)
                    param_store(to.address(base + run * to.stride + l), 0, to.bf16,
                                to.value(old[k], staged(run, l)));
            }
        }
    }
    tc_fence_before();
    if (ctas > 1)
        cluster_sync();              // nobody leaves while it is read
    else
        __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_free<1>(tmem, kTmemColumns);
}

}  // namespace

cudaError_t ortho_small_setup(int ctas, bool *fits) {
    static PerDevice known[5];
    const int d = PerDevice::device();
    int which = 0;
    while (1 << which < ctas) ++which;
    int v = known[which].get(d);
    if (!v) {
        cudaError_t e = cudaFuncSetAttribute(
            ortho_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes);
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(ortho_small_kernel,
                                     cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t c{};
        c.gridDim = dim3(ctas);
        c.blockDim = dim3(kThreads);
        c.dynamicSmemBytes = kSharedBytes;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim = {(unsigned)ctas, 1, 1};
        c.attrs = at;
        c.numAttrs = 1;
        int clusters = 0;
        e = cudaOccupancyMaxActiveClusters(&clusters, ortho_small_kernel, &c);
        if (e != cudaSuccess) {
            cudaGetLastError();
            clusters = 0;
        }
        v = clusters > 0 ? 2 : 1;
        known[which].set(d, v);
    }
    *fits = v == 2;
    return cudaSuccess;
}

cudaError_t launch_ortho_small(const OrthoArgs &a, int matrices, cudaStream_t stream) {
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)(matrices * a.small_ctas));
    c.blockDim = dim3(kThreads);
    c.dynamicSmemBytes = kSharedBytes;
    c.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {(unsigned)a.small_ctas, 1, 1};
    c.attrs = at;
    c.numAttrs = a.small_ctas > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&c, ortho_small_kernel, a);
}

}  // namespace aloco
