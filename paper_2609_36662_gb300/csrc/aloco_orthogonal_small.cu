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

// Matrices of the groups whose clusters have this launch's size.  Thread (row,
// half): columns half * 128 .. + 127 of its CTA's 256, of X in fp32 in registers;
// its fp16 values, A and P lie in shared memory as operands, K-major and MN-major
// in one.  Parts of A are added over the cluster in rank order.  A CTA whose wait
// runs out goes on with NaN, which its cluster gets with its part of A.
//
// A step is a chain of latencies (three products, their fences and reads, and the
// cluster's exchange: about 4 us, 6 with it), where kernels of their own take 20.
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
    for (uint32_t i = tid * 16; i < kXBytes + 2 * kABytes; i += kThreads * 16)
        store_shared(smem + i, make_uint4(0, 0, 0, 0));
    grid_go();
    grid_wait();

    // U, its norm, and the new momentum
    const Source s(args, g, matrix);
    const int j0 = half * kEach;
    const int count = r < m ? max(0, min(kEach, cols - j0)) : 0;  // of this thread
    float x[kEach];
    // (squares in fp32, where they fit: the SM adds two doubles a clock)
    float near = 0.f;
    double far = 0.0;
#pragma unroll
    for (int j = 0; j < kEach; j += 16) {
        float v[16];
        if (s.by4 && !g.tall && j + 16 <= count) {
            float4 q[4], o[4];
            const int64_t e = s.at + (int64_t)r * s.stride + first + j0 + j;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = load4(s.in, e + 4 * i, s.bf16);
            if (s.momentum) {
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = load4(s.momentum, e + 4 * i, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float *qi = &q[i].x, *oi = &o[i].x;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        oi[k] = s.mo.next(oi[k], qi[k]);
                        qi[k] = s.mo.u(oi[k], qi[k]);
                    }
                    *reinterpret_cast<float4 *>(s.momentum + e + 4 * i) = o[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[4 * i] = q[i].x;
                v[4 * i + 1] = q[i].y;
                v[4 * i + 2] = q[i].z;
                v[4 * i + 3] = q[i].w;
            }
        } else {
            // (element (r, c) of X is (c, r) of a tall matrix: lanes lie side by side)
            const int64_t step = g.tall ? s.stride : 1;
            const int64_t e = s.at + (g.tall ? (int64_t)(first + j0 + j) * s.stride + r
                                             : (int64_t)r * s.stride + first + j0 + j);
            float old[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool is = j + i < count;
                v[i] = is ? param_load(s.in, e + i * step, s.bf16) : 0.f;
                old[i] = is && s.momentum ? s.momentum[e + i * step] : 0.f;
            }
            if (s.momentum) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float next = s.mo.next(old[i], v[i]);
                    if (j + i < count) s.momentum[e + i * step] = next;
                    v[i] = s.mo.u(next, v[i]);
                }
            }
        }
        float sq = 0.f, top = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            sq = fmaf(v[i], v[i], sq);
            top = fmaxf(top, fabsf(v[i]));
            x[j + i] = v[i];
        }
        if (top < 1e18f && (top > 1e-12f || top == 0.f) && sq == sq) {
            near += sq;
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) far += (double)v[i] * (double)v[i];
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
        const bool usual = total > 1e-30 && total < 1e30;
        s_factor = usual ? kOrthoScale / (sqrtf((float)total) + (float)args.eps) : 0.f;
        if (!usual) s_sum[0] = (double)kOrthoScale / (sqrt(total) + args.eps);
    }
    __syncthreads();
    if (s_factor > 0.f) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) x[j] *= s_factor;
    } else {
        const double factor = s_sum[0];
#pragma unroll
        for (int j = 0; j < kEach; ++j) x[j] = (float)((double)x[j] * factor);
    }

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

    const Result to(args, g, gi, matrix);
    const int64_t step = g.tall ? to.stride : 1;
    const int64_t e = g.tall ? (int64_t)(first + j0) * to.stride + r
                             : (int64_t)r * to.stride + first + j0;
#pragma unroll
    for (int j = 0; j < kEach; j += 8) {
        if (!g.tall && to.whole && j + 8 <= count) {
            uint4 w[2];
            char *p = to.address(e + j);
            const int n = to.bf16 ? 1 : 2;
            for (int i = 0; i < n; ++i)
                w[i] = to.update ? reinterpret_cast<uint4 *>(p)[i] : make_uint4(0, 0, 0, 0);
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = x[j + i] * (1.f / kOrthoScale);
            if (to.bf16) {
                uint32_t *q = &w[0].x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __nv_bfloat162 h =
                        __floats2bfloat162_rn(to.value(__uint_as_float(q[i] << 16), o[2 * i]),
                                              to.value(__uint_as_float(q[i] & 0xffff0000u),
                                                       o[2 * i + 1]));
                    q[i] = *reinterpret_cast<const uint32_t *>(&h);
                }
                *reinterpret_cast<uint4 *>(p) = w[0];
            } else {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float *q = reinterpret_cast<float *>(&w[k]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) q[i] = to.value(q[i], o[4 * k + i]);
                    reinterpret_cast<uint4 *>(p)[k] = w[k];
                }
            }
            continue;
        }
        float old[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            old[i] = to.update && j + i < count
                         ? param_load(to.address(e + (j + i) * step), 0, to.bf16)
                         : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (j + i < count)
                param_store(to.address(e + (j + i) * step), 0, to.bf16,
                            to.value(old[i], x[j + i] * (1.f / kOrthoScale)));
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
