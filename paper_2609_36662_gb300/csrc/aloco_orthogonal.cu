// Orthogonal factors by Newton-Schulz products on the tensor cores: X <- (a +
// b A + c A A) X with A = X X^T, some steps of it, for many matrices at once.
//
// X in bf16 loses 1 to 4e-2 of the factor, in fp16 up to 0.15 at rank one: what
// multiplies X itself grows by a^steps where singular values are small.  So X is a sum
// of two fp16 values, of which products take the larger; the diagonal of the
// polynomial, which multiplies X itself, comes in fp32 from diagonals kept beside the
// matrices and takes both.
#include <climits>
#include <type_traits>

#include "aloco_orthogonal.cuh"
#include "aloco_tc.cuh"

namespace aloco {
namespace {

constexpr int kThreads = 256;        // of the norm and prepare kernels
constexpr int kEpilogueWarps = 8;
constexpr int kEpilogueWarp = 4;     // the first of them
constexpr int kProductThreads = 32 * (kEpilogueWarp + kEpilogueWarps);
constexpr int kHalfTile = 128;       // a CTA's rows of a tile
constexpr int kFull = 256;           // symmetric matrices' diagonal blocks that are whole
constexpr int kK = 64;               // k-elements of a slot: 128 bytes a row
constexpr int kBox = 64;             // rows of a copied box
constexpr int kBoxBytes = kBox * kK * 2;
constexpr int kSlotBytes = 4 * kBoxBytes;  // two boxes of either operand
constexpr int kSlots = 6;
constexpr int kStageBytes = 4096;    // an epilogue warp's: a pair of 32 x 32 fp16 blocks
constexpr int kSharedBytes =
    kSlots * kSlotBytes + kEpilogueWarps * kStageBytes + 1024 + 512;
constexpr int kRing = 4;             // tiles that a CTA knows of
constexpr int kAsk = 6;              // the next is taken so many slots before a tile's last

struct Work {
    int op;                          // of the group's list; < 0: there is no more
    int group, matrix;
    int row, col;                    // in tiles
    union {
        int before;                  // tiles of the matrix that have to be done
        int given_up;                // as it is told: they never were
    };
    int part;                        // of the depth
    int unused;
};
static_assert(sizeof(Work) == 32, "a ring's entry");

__device__ __forceinline__ const OrthoOp &op_of(const OrthoArgs &a, const Work &f) {
    return a.ops[a.g[f.group].list][f.op];
}
__device__ __forceinline__ int parts_of(const OrthoGroup &g, const OrthoOp &op) {
    return op.what == kUpdate ? 1 : g.split[op.what != kGram];
}

// Tiles in the order in which they are handed out: the first operation of all
// groups, the second of all, and so on.
struct Finder {
    int op = 0, group = 0, start = 0;

    // Tile t, not before an earlier one.
    __device__ __forceinline__ Work find(const OrthoArgs &a, int t, int tile) {
        Work f;
        for (;;) {
            const OrthoGroup &g = a.g[group];
            int n = 0;
            if (op < a.n_ops[g.list]) {
                const OrthoOp &o = a.ops[g.list][op];
                n = g.count * (o.what == kUpdate ? g.up_tiles : g.sym_tiles * parts_of(g, o));
            }
            if (t < start + n) break;
            start += n;
            if (++group == a.n_groups) group = 0, ++op;
        }
        f.op = op;
        f.group = group;
        const OrthoGroup &g = a.g[group];
        const OrthoOp &o = a.ops[g.list][op];
        t -= start;
        f.part = 0;
        if (o.what == kUpdate) {
            f.matrix = t / g.up_tiles;
            t -= f.matrix * g.up_tiles;
            const int rows = (g.m + tile - 1) / tile;
            f.col = t / rows;        // the left matrix's rows first: X's columns stay in L2
            f.row = t - f.col * rows;
        } else {
            const int parts = parts_of(g, o);
            f.matrix = t / (g.sym_tiles * parts);
            t -= f.matrix * g.sym_tiles * parts;
            f.part = t % parts;
            t /= parts;
            // row r of the lower triangle holds tiles r (r + 1) / 2 ..
            int r = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
            while (r * (r + 1) / 2 > t) --r;
            while ((r + 1) * (r + 2) / 2 <= t) ++r;
            f.row = r;
            f.col = t - r * (r + 1) / 2;
        }
        f.before = o.syms * g.sym_tiles + o.ups * g.up_tiles;
        return f;
    }
};

// A 32 x 32 block of fp16 values in a warp's shared memory: 64 bytes a row, whose
// 16-byte pieces are turned so that neither a row to a lane nor four lanes to a
// row meet in a bank.
__device__ __forceinline__ uint4 *piece(char *block, int row, int q) {
    return reinterpret_cast<uint4 *>(block) + row * 4 + (q ^ ((row >> 1) & 3));
}

// The block's pieces in global memory, four lanes to a row: 16-byte accesses of
// whole 64-byte stretches.  Rows and columns beyond the limits are not touched
// (columns up to the next multiple of 8 are padding).
struct Pieces {
    uint4 q[4];
    __device__ __forceinline__ void load(const __half *p, int64_t ld, int rows, int cols) {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + lane / 4, c = lane % 4 * 8;
            // (past the SM's cache: other SMs write it while this kernel runs)
            q[i] = r < rows && c < cols
                       ? __ldcg(reinterpret_cast<const uint4 *>(p + r * ld + c))
                       : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void to_shared(char *block) const {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int i = 0; i < 4; ++i) *piece(block, 8 * i + lane / 4, lane % 4) = q[i];
    }
};
__device__ __forceinline__ void store_block(char *block, __half *p, int64_t ld, int rows,
                                            int cols) {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + lane / 4, c = lane % 4 * 8;
        const uint4 q = *piece(block, r, lane % 4);
        if (r < rows && c < cols) *reinterpret_cast<uint4 *>(p + r * ld + c) = q;
    }
}

// Row `lane` in v.
__device__ __forceinline__ void rows_to_shared(char *block, const float (&v)[32]) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *piece(block, threadIdx.x % 32, q) =
            make_uint4(pack(v[8 * q], v[8 * q + 1]), pack(v[8 * q + 2], v[8 * q + 3]),
                       pack(v[8 * q + 4], v[8 * q + 5]), pack(v[8 * q + 6], v[8 * q + 7]));
}

// A 32 x 32 block at (r0, c0) of a symmetric matrix, row `lane` in v: as it lies,
// and mirrored if asked.
__device__ __forceinline__ void store_symmetric(__half *o, int m, int ld, int r0, int c0,
                                                bool mirrored, char *st, const float (&v)[32]) {
    const int lane = threadIdx.x % 32;
    __half *mirror = reinterpret_cast<__half *>(st + 2048);
    __syncwarp();
    rows_to_shared(st, v);
    if (mirrored) {
        // element (lane, c) to row c of the mirrored block
#pragma unroll
        for (int c = 0; c < 32; ++c) {
            const int q = (lane >> 3) ^ ((c >> 1) & 3);
            mirror[c * 32 + q * 8 + (lane & 7)] = __float2half_rn(v[c]);
        }
    }
    __syncwarp();
    store_block(st, o + (int64_t)r0 * ld + c0, ld, m - r0, ld - c0);
    if (mirrored) store_block(st + 2048, o + (int64_t)c0 * ld + r0, ld, m - c0, ld - r0);
}

// A 32 x 32 block of parameters, row by row as memory has it, in 16-byte pieces:
// fetched while the products run, joined with the factor in a warp's shared
// memory, and stored.
template <bool kBf16>
struct Param {
    static constexpr int kPieces = kBf16 ? 4 : 8, kEach = kBf16 ? 8 : 4;
    uint4 q[kPieces];
    static __device__ __forceinline__ int row(int i) {
        return i * (32 / kPieces) + (int)(threadIdx.x % 32) / kPieces;
    }
    static __device__ __forceinline__ int col() { return threadIdx.x % kPieces * kEach; }
    static __device__ __forceinline__ uint4 *place(char *st, int r, int c) {
        return kBf16 ? piece(st, r, c / kEach)
                     : reinterpret_cast<uint4 *>(st) + r * 8 + ((c / kEach) ^ (r & 7));
    }
    // (y, x): the block's place in memory's rows and columns
    __device__ __forceinline__ void load(const Result &to, int y, int x, int rows, int cols) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int r = y + row(i), c = x + col();
            q[i] = r < rows && c < cols
                       ? *reinterpret_cast<const uint4 *>(to.address(r * to.stride + c))
                       : make_uint4(0, 0, 0, 0);
        }
    }
    // v: row `lane` of X's block
    __device__ __forceinline__ void join(const Result &to, char *st, const float (&v)[32]) const {
        const int lane = threadIdx.x % 32;
        __syncwarp();
        if (to.update) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) *place(st, row(i), col()) = q[i];
            __syncwarp();
        }
        if (to.tall) {               // memory's rows are X's columns
#pragma unroll
            for (int c = 0; c < 32; ++c) {
                char *at = reinterpret_cast<char *>(place(st, c, lane)) + lane % kEach * (16 / kEach);
                param_store(at, 0, kBf16,
                            to.value(to.update ? param_load(at, 0, kBf16) : 0.f, v[c]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; i += kEach) {
                uint4 *at = place(st, lane, i), w = to.update ? *at : make_uint4(0, 0, 0, 0);
                uint32_t *p = &w.x;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (kBf16) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(
                            to.value(__uint_as_float(p[j] << 16), v[i + 2 * j]),
                            to.value(__uint_as_float(p[j] & 0xffff0000u), v[i + 2 * j + 1]));
                        p[j] = *reinterpret_cast<const uint32_t *>(&h);
                    } else {
                        p[j] = __float_as_uint(to.value(__uint_as_float(p[j]), v[i + j]));
                    }
                }
                *at = w;
            }
        }
        __syncwarp();
    }
    static __device__ __forceinline__ void store(const Result &to, char *st, int y, int x,
                                                 int rows, int cols) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int r = y + row(i), c = x + col();
            const uint4 w = *place(st, row(i), col());
            if (r < rows && c < cols)
                *reinterpret_cast<uint4 *>(to.address(r * to.stride + c)) = w;
        }
    }
};

// The same value by value, where pieces are not aligned.
template <bool kBf16>
__device__ __forceinline__ void store_values(const Result &to, int y, int x, int rows, int cols,
                                             char *st, const float (&v)[32]) {
    const int lane = threadIdx.x % 32;
    float *f = reinterpret_cast<float *>(st);
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 32; ++c) {
        const int r = to.tall ? c : lane, e = to.tall ? lane : c;
        f[r * 32 + (e ^ r)] = v[c];
    }
    __syncwarp();
    const bool in = x + lane < cols;
#pragma unroll
    for (int r = 0; r < 32; r += 8) {
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool is = in && y + r + j < rows;
            const float o = f[(r + j) * 32 + (lane ^ (r + j))];
            w[j] = to.value(is && to.update
                                ? param_load(to.address((y + r + j) * to.stride + x + lane), 0, kBf16)
                                : 0.f,
                            o);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (in && y + r + j < rows)
                param_store(to.address((y + r + j) * to.stride + x + lane), 0, kBf16, w[j]);
    }
}

// Where tiles that a matrix's next products take are done with: what `count` warps
// have written is seen by whoever finds them counted.  A matrix of which a tile was
// given up has kLost there, which no count reaches: a count says how much is done, not
// what, so that tiles without their operands must not make up for others.
constexpr int kLost = 1 << 30;
__device__ __forceinline__ int load_acquire(const int *p) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ bool wait_done(const int *done, int count, const volatile int *abort) {
    int is = load_acquire(done);
    if (is < count) {
        const long long t0 = clock64();
        while ((is = load_acquire(done)) < count) {
            if (*abort || clock64() - t0 > kTmaWaitCycles) return false;
            __nanosleep(64);
        }
    }
    return is < kLost;
}
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok) return true;
        if (clock64() - t0 > 2 * kTmaWaitCycles) return false;
    }
}

// All operations of all matrices, tile by tile.  CTAs (pairs of them) take the next
// tile when they have asked for the operands of the one before, so that no two
// wait for each other: what a tile needs was handed out before it, and counts of
// the matrix's blocks that are done say when it is there.
//
// In a CTA two threads copy operands into a ring of slots, one issues the products
// into one of two accumulators, eight warps join the other one with what it needs
// and write it, and one (of a pair's first CTA) takes the tiles, waits for what they
// need, and tells the others.  Of symmetric matrices the lower tiles are computed
// and kept, with whole blocks of kFull on the diagonal; where a product needs what
// would lie above them it takes the tile below, MN-major instead of K-major.
//
// Bound by the tensor cores where matrices are large (16 x 2048 x 2048: 512 of 540
// cycles a slot, at the clock that 1360 W leave); at 768 by the epilogue too, which
// moves 8 bytes an element of X in and out of L2 for 12 slots of products (48 x 768
// x 768: tensor cores 43 % busy, HBM 44 % of its peak, 7.8 GB through L2; 593 us the
// whole call on matrices that are not in L2, 567 where they are the last call's); for a
// few small matrices by 15 dependent products, of which each takes about 10 us: 1 until
// it is known that its operands are there, 2 until the first of them have come, 3 of
// products, 4 until the last tile is written.
// When it came a kernel for every product took 315 us in place of 254 for 7 odd matrices
// of 3 workers, 663 of 641 for 48 x 768 x 768 and 2.48 of 2.25 ms for 16 x 2048 x 2048: a
// matrix waits for itself alone.
//
// A wait that runs out ends the waits of its pair.  The tiles that the pair knows of
// become NaN, and their matrices are marked: whoever takes another tile of one does
// the same, without a wait.  The pair takes no more tiles, unless all pairs have given
// up: then the last of them makes NaN of what is left, so that nothing stays unwritten.
template <int kCtas, bool kOutBf16, bool kParts>
__global__ void __launch_bounds__(kProductThreads, 1)
    ortho_chain_kernel(const __grid_constant__ OrthoArgs args) {
    constexpr int kTile = kHalfTile * kCtas;
    constexpr uint32_t kDesc = product_desc(kTile, kTile);
    constexpr int kPlaces = kCtas * kEpilogueWarps;      // warps that share a tile
    constexpr int kBlocks = kTile / 64;                  // of a warp: 32 x 32 of its tile
    constexpr int kSignals = kPlaces * kBlocks;
    extern __shared__ char raw[];
    const uint32_t smem = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t bars = smem + kSlots * kSlotBytes + kEpilogueWarps * kStageBytes;
    const auto full = [&](int s) { return bars + 8 * s; };
    const auto empty = [&](int s) { return bars + 8 * (kSlots + s); };
    const auto acc_full = [&](int s) { return bars + 8 * (2 * kSlots + s); };
    const auto acc_empty = [&](int s) { return bars + 8 * (2 * kSlots + 2 + s); };
    const uint32_t drained = bars + 8 * (2 * kSlots + 4);
    const auto told = [&](int s) { return bars + 8 * (2 * kSlots + 5 + s); };
    const auto heard = [&](int s) { return bars + 8 * (2 * kSlots + 5 + kRing + s); };
    const uint32_t asked = bars + 8 * (2 * kSlots + 5 + 2 * kRing);
    const auto work_at = [&](int s) { return ((asked + 8 + 15) & ~15u) + 32 * s; };
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;             // a wait of this CTA's, or its pair's, ran out
    __shared__ volatile int s_issued[2 * kCtas]; // slots that the copying threads have filled

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = kCtas == 1 ? 0 : cluster_rank();
    const int tiles = args.tiles;

    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(acc_full(s), 1);
            mbar_init(acc_empty(s), kEpilogueWarps * kCtas);
        }
        mbar_init(drained, 1);
        for (int s = 0; s < kRing; ++s) {
            mbar_init(told(s), 1);
            // all that hear of a tile: a CTA's copying threads and warps, and whoever
            // issues the products
            mbar_init(heard(s), kCtas * (kEpilogueWarps + 2) + 1);
        }
        mbar_init(asked, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_alloc<kCtas>(smem_addr(&s_tmem), 2 * kTile);
    if (warp == 4)
        for (int i = lane; i < kOrthoMaps * args.n_groups; i += 32)
            fetch_map(&args.map[i / args.n_groups][i % args.n_groups]);
    tc_fence_before();
    __syncthreads();
    if constexpr (kCtas == 2) cluster_sync();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    grid_go();
    grid_wait();

    // (to both CTAs of a pair)
    const auto tell_pair = [&](volatile int *at, int v) {
        *at = v;
        if constexpr (kCtas == 2)
            asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(
                             cluster_addr(smem_addr(const_cast<int *>(at)), rank ^ 1)),
                         "r"(v)
                         : "memory");
    };
    const auto give_up = [&] { tell_pair(&s_abort, 1); };

    // The next tile, as all but the thread that takes it hear of it.
    int ring = 0;
    uint32_t ring_phase = 0;
    const auto on = [&] {
        if (++ring == kRing) ring = 0, ring_phase ^= 1;
    };
    const auto hear = [&](bool whole_warp) -> Work {
        Work f;
        f.op = -1;
        if (mbar_wait_cluster(told(ring), ring_phase)) {
            asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(f.op), "=r"(f.group), "=r"(f.matrix), "=r"(f.row)
                         : "r"(work_at(ring))
                         : "memory");
            asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(f.col), "=r"(f.given_up), "=r"(f.part), "=r"(f.unused)
                         : "r"(work_at(ring) + 16)
                         : "memory");
        } else {
            give_up();
        }
        if (whole_warp) __syncwarp();
        if (!whole_warp || lane == 0) {
            if (kCtas == 1 || rank == 0)
                mbar_arrive(heard(ring));
            else
                asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                                 cluster_addr(heard(ring), 0))
                             : "memory");
        }
        on();
        return f;
    };
    const auto done_of = [&](const Work &f) { return args.g[f.group].done + f.matrix; };
    // the k-elements that a tile, or its part, takes: from *begin on
    const auto depth_of = [&](const Work &f, const OrthoOp &op, int *begin) {
        const OrthoGroup &g = args.g[f.group];
        const int all = op.what == kGram ? g.n : g.m, parts = kParts ? parts_of(g, op) : 1;
        const int chunks = (all + kK - 1) / kK;
        *begin = chunks * f.part / parts * kK;
        return min(all, chunks * (f.part + 1) / parts * kK);
    };

    if (warp == 2 && lane == 0 && rank == 0) {
        // Takes tiles, and tells of one when all that it needs is there.
        Finder finder;
        uint32_t asked_phase = 0;
        bool counted = false, last = false;
        for (;;) {
            if (s_abort && !counted) {
                counted = true;
                last = atomicAdd(args.next_tile + 1, 1) + 1 == (int)gridDim.x / kCtas;
            }
            const int next = counted && !last ? tiles : atomicAdd(args.next_tile, 1);
            Work f;
            f.op = -1;
            if (next < tiles) {
                f = finder.find(args, next, kTile);
                f.given_up = s_abort || !wait_done(done_of(f), f.before * kSignals, &s_abort);
            }
            if (!mbar_wait_cluster(heard(ring), ring_phase ^ 1)) {
                give_up();
                break;
            }
            for (int p = 0; p < kCtas; ++p) {
                const uint32_t at = kCtas == 1 ? work_at(ring) : cluster_addr(work_at(ring), p);
                asm volatile("st.shared::cluster.v4.s32 [%0], {%1, %2, %3, %4};" ::"r"(at),
                             "r"(f.op), "r"(f.group), "r"(f.matrix), "r"(f.row)
                             : "memory");
                asm volatile("st.shared::cluster.v4.s32 [%0], {%1, %2, %3, %4};" ::"r"(at + 16),
                             "r"(f.col), "r"(f.given_up), "r"(f.part), "r"(0)
                             : "memory");
            }
            mbar_arrive(told(ring));
            if constexpr (kCtas == 2)
                asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                                 cluster_addr(told(ring), 1))
                             : "memory");
            on();
            if (f.op < 0) break;
            if (!mbar_wait_cluster(asked, asked_phase)) {
                give_up();
                break;
            }
            asked_phase ^= 1;
        }
    } else if ((warp == 0 || warp == 3) && lane == 0) {
        // One thread for either operand: copying both, a thread takes as long as
        // the products of a slot do.
        const bool is_b = warp == 3, leads = rank == 0 && !is_b;
        const uint32_t bar0 = kCtas == 1 ? full(0) : cluster_addr(full(0), 0);
        int slot = 0, issued = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (;;) {
            const Work f = hear(false);
            if (f.op < 0) break;
            if (f.given_up) {
                if (leads) mbar_arrive(asked);
                continue;
            }
            const OrthoOp &op = op_of(args, f);
            int begin;
            const int end = depth_of(f, op, &begin);
            const int ask = begin + max(0, (end - begin - 1) / kK + 1 - kAsk) * kK;
            ok = ok && !s_abort;
            // operands were written by ordinary stores
            asm volatile("fence.proxy.async;" ::: "memory");
            const bool x = op.what == kGram || (op.what == kUpdate && is_b);
            const CUtensorMap *map =
                &args.map[x ? kMapX0 + op.x : kMapSym + (is_b ? op.right : op.left)][f.group];
            const int row = (is_b ? f.col : f.row) * kTile + (int)rank * kHalfTile;
            // columns from here on lie below, MN-major (X does throughout)
            const int turn = op.what == kGram ? INT_MAX : x ? 0 : (row / kFull + 1) * kFull;
            for (int c = begin; c < end; c += kK) {
                if (leads && c == ask) mbar_arrive(asked);
                if (!ok || !(ok = mbar_wait(empty(slot), phase ^ 1, &s_abort))) continue;
                const uint32_t at = smem + slot * kSlotBytes + (is_b ? 2 * kBoxBytes : 0);
                const uint32_t bar = bar0 + 8 * slot;
                if (leads) mbar_arrive_expect_tx(full(slot), kCtas * kSlotBytes);
                if (args.test_stall1 == 0 || blockIdx.x != 0 || issued != args.test_stall1 - 1) {
                    if (c < turn) {
                        tensor_load<kCtas>(at, map, c, row, f.matrix, bar);
                        tensor_load<kCtas>(at + kBoxBytes, map, c, row + kBox, f.matrix, bar);
                    } else {
                        tensor_load<kCtas>(at, map, row, c, f.matrix, bar);
                        tensor_load<kCtas>(at + kBoxBytes, map, row + kBox, c, f.matrix, bar);
                    }
                }
                ++issued;
                if (++slot == kSlots) slot = 0, phase ^= 1;
            }
            if (!ok) give_up();
        }
        tell_pair(&s_issued[2 * rank + is_b], issued);
    } else if (warp == 1 && lane == 0 && rank == 0) {
        int slot = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        bool ok = true;
        for (;;) {
            const Work f = hear(false);
            if (f.op < 0) break;
            if (f.given_up) continue;
            const OrthoOp &op = op_of(args, f);
            int begin;
            const int end = depth_of(f, op, &begin);
            if (ok) ok = mbar_wait(acc_empty(acc), acc_phase ^ 1, &s_abort);
            tc_fence_after();
            const int turn_a = op.what == kGram ? INT_MAX : (f.row * kTile / kFull + 1) * kFull;
            const int turn_b = op.what == kGram     ? INT_MAX
                               : op.what == kUpdate ? 0
                                                    : (f.col * kTile / kFull + 1) * kFull;
            const uint32_t d = tmem + acc * kTile;
            for (int k = begin; ok && k < end; k += kK) {
                if (!(ok = mbar_wait(full(slot), phase, &s_abort))) break;
                tc_fence_after();
                const uint32_t a0 = smem + slot * kSlotBytes, b0 = a0 + 2 * kBoxBytes;
                const bool ta = k >= turn_a, tb = k >= turn_b;
                const uint32_t desc = kDesc | (ta ? kAMnMajor : 0) | (tb ? kBMnMajor : 0);
                const uint64_t da = operand_desc(a0, ta ? kBoxBytes : 16);
                const uint64_t db = operand_desc(b0, tb ? kBoxBytes : 16);
                // 16 k-elements on, in 16 bytes: 32 bytes of a row, or 16 rows
                const int na = ta ? 2048 / 16 : 2, nb = tb ? 2048 / 16 : 2;
                // (straight on: between products this thread has 128 cycles)
                product<kCtas>(d, da, db, desc, k != begin);
                if (end - k > 16) product<kCtas>(d, da + na, db + nb, desc, true);
                if (end - k > 32) product<kCtas>(d, da + 2 * na, db + 2 * nb, desc, true);
                if (end - k > 48) product<kCtas>(d, da + 3 * na, db + 3 * nb, desc, true);
                product_commit<kCtas>(empty(slot));
                if (++slot == kSlots) slot = 0, phase ^= 1;
            }
            if (ok)
                product_commit<kCtas>(acc_full(acc));
            else
                give_up();
            if (acc) acc_phase ^= 1;
            acc ^= 1;
        }
    } else if (warp >= kEpilogueWarp) {
        // a warp reads its quarter of the lanes, and half of the columns
        const int quad = warp % 4, half = (warp - kEpilogueWarp) / 4;
        char *st = raw + (smem - smem_addr(raw)) + kSlots * kSlotBytes +
                   (warp - kEpilogueWarp) * kStageBytes;
        int acc = 0;
        uint32_t acc_phase = 0;
        for (;;) {
            const Work f = hear(true);
            if (f.op < 0) break;
            const OrthoGroup &g = args.g[f.group];
            const OrthoOp &op = op_of(args, f);
            const bool up = op.what == kUpdate;
            const int m = g.m, r0 = f.row * kTile + (int)rank * kHalfTile + quad * 32;
            const int r = r0 + lane, limit = up ? g.n : m;
            const int c_end = min(limit, f.col * kTile + (half + 1) * (kTile / 2));
            int c0 = f.col * kTile + half * (kTile / 2);
            const bool some = r0 < m && c0 < c_end;
            const int64_t row0 = (int64_t)f.matrix * m;  // of the matrix, in its group
            // (single CTAs have two tiles of a block on the diagonal to fill)
            const bool mirrored = kCtas == 1 && f.row != f.col &&
                                  f.row * kTile / kFull == f.col * kTile / kFull;
            const float ca = args.coef[op.step][0], cb = args.coef[op.step][1],
                        cc = args.coef[op.step][2];
            // a + b L + c L^2 = c (L + e)^2 + a - c e^2 with e = b / 2c, which is added to
            // L's diagonal: its tiles need nothing but their product
            const float shift = op.shifted ? cb / (2.f * cc) : 0.f;
            const bool joined = op.what == kPoly && !op.shifted;   // b L is added
            const int parts = kParts ? parts_of(g, op) : 1;
            const bool in_parts = kParts && parts > 1;
            // what a product is joined with: of L whole rows, of X also blocks that lie
            // as this warp holds them; fetched a block ahead
            uint4 *rest = g.rest + ((int64_t)(f.matrix * g.blocks_down + r0 / 32) * g.blocks_across +
                                    c0 / 32) * kBlockPieces + lane;
            const Result to(args, g, f.group, f.matrix);
            Pieces part;
            uint4 lo[4];
            float by_row = 0.f, by_row2 = 0.f;
            const int begin = c0;
            const auto fetch_l = [&](int c) {
                part.load(g.sym[op.left] + (row0 + r0) * g.lda + c, g.lda, m - r0, m - c);
            };
            const auto fetch_x = [&](int c) {
                const uint4 *p = rest + (c - begin) / 32 * kBlockPieces;
#pragma unroll
                for (int i = 0; i < 4; ++i) lo[i] = __ldcg(p + 32 * i);
                part.load(g.x[op.x] + (row0 + r0) * g.ldx + c, g.ldx, m - r0, g.n - c);
            };
            if (op.last && some && to.update) {
                // parameters come from far: to L2 while the products run
                const int along = to.tall ? 32 : c_end - c0, down = to.tall ? c_end - c0 : 32;
                for (int i = lane; i < down; i += 32) {
                    const int y = (to.tall ? c0 : r0) + i, x = to.tall ? r0 : c0;
                    if (y >= g.rows) break;
                    for (int j = 0; j < along && x + j < g.cols; j += 32)
                        fetch_l2(to.address(y * to.stride + x + j));
                }
            }
            bool ok = !s_abort && !f.given_up;
            if (op.what != kGram && some) {
                if (r < m) {
                    by_row = __ldcg(g.diag[op.left] + row0 + r);
                    if (op.what == kProduct) by_row2 = __ldcg(g.diag[op.right] + row0 + r);
                }
                if (up) {
                    // what is kept of X beside the operands comes to L2 while the
                    // products run
                    const int lines = (c_end - c0 + 31) / 32 * 16;
                    for (int i = lane; i < lines; i += 32) fetch_l2(rest - lane + 8 * i);
                    fetch_x(c0);
                } else if (joined && !in_parts) {
                    fetch_l(c0);
                }
            }
            if (ok) ok = mbar_wait(acc_full(acc), acc_phase, &s_abort);
            ok = __all_sync(~0u, ok);
            if (!ok && !f.given_up) give_up();
            tc_fence_after();
            // the accumulator goes back when the last block has been read (a tile that was
            // given up has none)
            const auto release = [&] {
                if (f.given_up) return;
                tc_fence_before();
                __syncwarp();
                if (lane) return;
                if (kCtas == 1)
                    mbar_arrive(acc_empty(acc));
                else
                    mbar_arrive_cluster(cluster_addr(acc_empty(acc), 0));
            };
            // Of a tile in parts the warps that share a place go through its halves in turn,
            // every other one from the second half on: where another part is missing a
            // warp leaves its sums, where all others are there it finishes the half.  So
            // two parts that end together finish a half each, and nobody waits.  (One warp
            // that finishes all: 11 us after the last product of 2048 rows.)
            const int64_t tile =
                (int64_t)f.matrix * g.sym_tiles + f.row * (f.row + 1) / 2 + f.col;
            const int place = (int)rank * kEpilogueWarps + warp - kEpilogueWarp;
            const int64_t next_part = kPlaces * kBlocks * kBlockQuads;
            float4 *const sums = in_parts
                                     ? g.sums + tile * max(g.split[0], g.split[1]) * next_part +
                                           place * kBlocks * kBlockQuads + lane
                                     : nullptr;
            const auto read = [&](int c, uint32_t (&u)[32]) {
                __syncwarp();
                tmem_read32(tmem + acc * kTile + (c - f.col * kTile) + (quad << 21), u);
                if (!ok) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) u[i] = 0x7fffffff;
                }
            };
            // Columns [c, to): true if all other parts' sums are there.
            const auto meets = [&](bool late, int half, int c, int to) {
                int *count = g.came + (tile * kPlaces + place) * 2 + half;
                int came = late && lane == 0 ? load_acquire(count) : 0;
                if (__shfl_sync(~0u, came, 0) != parts - 1) {
                    float4 *at = sums + f.part * next_part + (c - begin) / 32 * kBlockQuads;
#pragma unroll 1
                    for (; c < to; c += 32, at += kBlockQuads) {
                        uint32_t u[32];
                        read(c, u);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            at[32 * i] = make_float4(
                                __uint_as_float(u[4 * i]), __uint_as_float(u[4 * i + 1]),
                                __uint_as_float(u[4 * i + 2]), __uint_as_float(u[4 * i + 3]));
                    }
                    __syncwarp();
                    if (lane == 0)
                        asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;"
                                     : "=r"(came)
                                     : "l"(count)
                                     : "memory");
                    if (__shfl_sync(~0u, came, 0) != parts - 1) return false;
                }
                if (lane == 0) *count = 0;   // for the next product
                __syncwarp();
                return true;
            };
            // column c0's sums of this row
            const auto values = [&](float (&v)[32]) {
                uint32_t u[32];
                read(c0, u);
                if (c0 + 32 >= c_end) release();
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(u[i]);
            };
            // The same of all parts: of two this warp's and the other's, of more all as
            // they lie there, in their order.
            const auto total = [&](float (&v)[32]) {
                uint32_t u[32];
                read(c0, u);
                const float4 *p = sums + (c0 - begin) / 32 * kBlockQuads;
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = parts == 2 ? __uint_as_float(u[i]) : 0.f;
#pragma unroll 1
                for (int k = 0; k < parts; ++k, p += next_part) {
                    if (parts == 2 && k == f.part) continue;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float4 q = __ldcg(p + 32 * i);
                        v[4 * i] += q.x;
                        v[4 * i + 1] += q.y;
                        v[4 * i + 2] += q.z;
                        v[4 * i + 3] += q.w;
                    }
                }
            };
            int finished = kBlocks;          // blocks
            if (!some) {
                release();
                if (f.part) finished = 0;
            } else if (!up) {
                const float scale = op.what == kGram   ? 1.f / (kOrthoScale * kOrthoScale)
                                    : op.what == kPoly ? cc
                                                       : 1.f;
                __half *out = g.sym[op.out] + row0 * g.lda;
                int stop = c_end;
                // (of blocks that there are not the first part tells)
                if (in_parts) finished = f.part ? 0 : kBlocks - (c_end - begin + 31) / 32;
#pragma unroll 1
                for (int turn = 0; turn < (in_parts ? 2 : 1); ++turn) {
                    if (in_parts) {
                        const int half = turn ^ (f.part & 1);
                        c0 = begin + half * (kTile / 4);
                        stop = min(c_end, c0 + kTile / 4);
                        if (c0 >= stop || !meets(turn && parts == 2, half, c0, stop)) continue;
                        finished += (stop - c0 + 31) / 32;
                        if (joined) fetch_l(c0);
                    }
#pragma unroll 1
                    for (; c0 < stop; c0 += 32) {
                        float v[32];
                        if (in_parts)
                            total(v);
                        else
                            values(v);
                        if (joined) {
                            __syncwarp();
                            part.to_shared(st);
                            if (c0 + 32 < stop) fetch_l(c0 + 32);
                            __syncwarp();
                        }
                        // The diagonal from what lies beside the operands: their own values as
                        // the product has them are taken out, and put back unrounded.
                        float own = 0.f;
                        if (c0 == r0) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (i == lane) own = v[i];
                            const auto rounded = [](float x) {
                                return __half2float(__float2half_rn(x));
                            };
                            if (op.what == kGram) {
                                own *= scale;
                            } else if (op.what == kPoly) {
                                const float s = rounded(by_row + shift);
                                own = ca + cb * by_row + cc * (by_row * by_row + (own - s * s));
                            } else {
                                own = by_row * by_row2 +
                                      (own - rounded(by_row) * rounded(by_row2));
                            }
                            if (r < m) g.diag[op.out][row0 + r] = own;
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] *= scale;
                        if (joined) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint4 w = *piece(st, lane, i);
                                const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const float2 h = unpack(ws[j]);
                                    v[8 * i + 2 * j] = fmaf(cb, h.x, v[8 * i + 2 * j]);
                                    v[8 * i + 2 * j + 1] = fmaf(cb, h.y, v[8 * i + 2 * j + 1]);
                                }
                            }
                        }
                        if (c0 == r0) {
                            const float kept =
                                op.bare ? 0.f : op.what == kGram ? own + shift : own;
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (i == lane) v[i] = kept;
                        }
                        store_symmetric(out, m, g.lda, r0, c0, mirrored, st, v);
                    }
                }
                if (in_parts) release();
            } else {
#pragma unroll 1
                for (; c0 < c_end; c0 += 32) {
                    Param<kOutBf16> param;
                    const int y = to.tall ? c0 : r0, x = to.tall ? r0 : c0;
                    if (op.last && to.update && to.whole) param.load(to, y, x, g.rows, g.cols);
                    float v[32];
                    values(v);
                    __syncwarp();
                    part.to_shared(st);
                    uint32_t ls[16];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        ls[4 * i] = lo[i].x;
                        ls[4 * i + 1] = lo[i].y;
                        ls[4 * i + 2] = lo[i].z;
                        ls[4 * i + 3] = lo[i].w;
                    }
                    if (c0 + 32 < c_end) fetch_x(c0 + 32);
                    __syncwarp();
                    uint4 w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = *piece(st, lane, i);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t hs = i % 4 == 0   ? w[i / 4].x
                                            : i % 4 == 1 ? w[i / 4].y
                                            : i % 4 == 2 ? w[i / 4].z
                                                         : w[i / 4].w;
                        const float2 h = unpack(hs), l = unpack(ls[i]);
                        v[2 * i] = fmaf(by_row, h.x, fmaf(by_row, l.x, v[2 * i]));
                        v[2 * i + 1] = fmaf(by_row, h.y, fmaf(by_row, l.y, v[2 * i + 1]));
                    }
                    if (op.last) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] *= 1.f / kOrthoScale;
                        if (to.whole) {
                            param.join(to, st, v);
                            param.store(to, st, y, x, g.rows, g.cols);
                        } else {
                            store_values<kOutBf16>(to, y, x, g.rows, g.cols, st, v);
                        }
                        continue;
                    }
                    uint4 *p = rest + (c0 - begin) / 32 * kBlockPieces;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t h[4], l[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float x0 = v[8 * i + 2 * j], x1 = v[8 * i + 2 * j + 1];
                            h[j] = pack(x0, x1);
                            const float2 b = unpack(h[j]);
                            l[j] = pack(x0 - b.x, x1 - b.y);
                        }
                        *piece(st, lane, i) = make_uint4(h[0], h[1], h[2], h[3]);
                        p[32 * i] = make_uint4(l[0], l[1], l[2], l[3]);
                    }
                    __syncwarp();
                    store_block(st, g.x[op.x ^ 1] + (row0 + r0) * g.ldx + c0, g.ldx, m - r0,
                                g.n - c0);
                }
            }
            if (!ok && lane == 0) atomicMax(done_of(f), kLost);
            if (!op.last && finished) {
                // done: what this warp has written is seen behind the count (by tensor
                // copies behind a fence of theirs)
                __syncwarp();
                if (lane == 0)
                    asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(done_of(f)),
                                 "r"(finished)
                                 : "memory");
            }
            if (f.given_up) continue;
            if (acc) acc_phase ^= 1;
            acc ^= 1;
        }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (kCtas == 2) cluster_sync();
    tc_fence_after();
    if (s_abort) {
        // All threads of the pair are behind their loops here, wherever each of them gave
        // up: what is in flight lands before shared memory and accumulators go back.
        if ((warp == 0 || warp == 3) && lane == 0) {
            const bool is_b = warp == 3, leads = rank == 0 && !is_b;
            const uint32_t bar0 = kCtas == 1 ? full(0) : cluster_addr(full(0), 0);
            const int issued = s_issued[2 * rank + is_b];
            // A slot that not all copying threads have filled is free in both CTAs (one of
            // them has seen that): the others fill it too, so that it completes.
            const auto fill = [&](int i) {
                const uint32_t at = smem + i % kSlots * kSlotBytes + (is_b ? 2 * kBoxBytes : 0);
                for (int k = 0; k < 2; ++k)
                    tensor_load<kCtas>(at + k * kBoxBytes, &args.map[kMapX0][0], 0, 0, 0,
                                       bar0 + 8 * (i % kSlots));
            };
            // (what the testing hook left out)
            if (blockIdx.x == 0 && args.test_stall1 > 0 && args.test_stall1 <= issued)
                fill((int)args.test_stall1 - 1);
            int last = 0;
            for (int k = 0; k < 2 * kCtas; ++k) last = max(last, s_issued[k]);
            for (int i = issued; i < last; ++i) {
                if (leads) mbar_arrive_expect_tx(full(i % kSlots), kCtas * kSlotBytes);
                fill(i);
            }
            if (leads)               // each slot's last use
                for (int i = max(0, last - kSlots); i < last; ++i)
                    mbar_wait(full(i % kSlots), (i / kSlots) & 1, nullptr);
        } else if (warp == 1 && lane == 0 && rank == 0) {
            product_commit<kCtas>(drained);
            mbar_wait(drained, 0, nullptr);
        }
        __syncthreads();
        if constexpr (kCtas == 2) cluster_sync();
    }
    if (warp == 2) tmem_free<kCtas>(tmem, 2 * kTile);
}

// The block's sum, in thread 0.
__device__ __forceinline__ double block_sum(double s, double *shared) {
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = s;
    __syncthreads();
    s = 0.0;
    if (threadIdx.x == 0)
        for (int i = 0; i < (int)blockDim.x / 32; ++i) s += shared[i];
    return s;
}

// Sums of squares of the matrices' stretches.
__global__ void __launch_bounds__(kThreads)
    ortho_norm_kernel(const __grid_constant__ OrthoArgs args) {
    __shared__ double shared[kThreads / 32];
    grid_go();
    grid_wait();
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < args.counters;
         i += gridDim.x * kThreads)
        args.next_tile[i] = 0;       // for the products' kernel
    const int gi = find_group(args, blockIdx.x, [](const OrthoGroup &g) { return g.norm0; });
    const OrthoGroup &g = args.g[gi];
    const int b = blockIdx.x - g.norm0, matrix = b / g.chunks, chunk = b - matrix * g.chunks;
    const Source s(args, g, matrix);
    const int64_t total = (int64_t)g.rows * g.cols;
    const int64_t begin = (int64_t)chunk * g.chunk;
    const int n = (int)min((int64_t)g.chunk, total - begin);   // begin: a multiple of 4
    // (a chunk of a matrix with padded rows starts in row r0, column c0)
    const int64_t r0 = begin / g.cols;
    const int c0 = (int)(begin - r0 * g.cols);
    const bool solid = s.stride == g.cols;
    const auto place = [&](int i) -> int64_t {
        if (solid) return begin + i;
        const unsigned c = (unsigned)c0 + (unsigned)i, r = c / (unsigned)g.cols;
        return (r0 + r) * s.stride + (c - r * (unsigned)g.cols);
    };
    double sum = 0.0;
    float v[16];
    if (s.by4) {
        for (int i = 4 * threadIdx.x; i < n; i += 16 * kThreads) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int e = i + j * 4 * kThreads;
                const float4 x = e < n ? s.u4(place(e)) : make_float4(0.f, 0.f, 0.f, 0.f);
                v[4 * j] = x.x;
                v[4 * j + 1] = x.y;
                v[4 * j + 2] = x.z;
                v[4 * j + 3] = x.w;
            }
            sum += squares(v);
        }
    } else {
        for (int i = threadIdx.x; i < n; i += 16 * kThreads) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int e = i + j * kThreads;
                v[j] = e < n ? s.u(place(e)) : 0.f;
            }
            sum += squares(v);
        }
    }
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) g.partial[(int64_t)matrix * g.chunks + chunk] = sum;
}

constexpr int kPrep = 64;            // rows and columns of a prepared tile

// X = U 2^8 / (|U| + eps) as a sum of two fp16 values, transposed where the matrix
// is tall, and the new momentum.  Bound by HBM: 48 x 768 x 768 fp32 (227 MB) 51 us
// with cold caches.  Five blocks an SM (48 registers, of which it spills 24 bytes): 4 us
// less than four or six in a call.
__global__ void __launch_bounds__(kThreads, 5)
    ortho_prepare_kernel(const __grid_constant__ OrthoArgs args) {
    __shared__ float s_f;            // the factor, where fp32 does for it
    __shared__ double s_factor;
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
    const Source s(args, g, matrix);
    const int tx = threadIdx.x % 16 * 4, ty = threadIdx.x / 16;

    // (the values first: they do not wait for the norm)
    float4 in[4], old[4];
    if (s.by4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + ty + 16 * i, c = c0 + tx;
            const bool is = r < g.rows && c < g.cols;
            const int64_t e = s.at + r * s.stride + c;
            in[i] = is ? load4(s.in, e, s.bf16) : make_float4(0.f, 0.f, 0.f, 0.f);
            old[i] = is && s.momentum ? load4(s.momentum, e, 0) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    // (few warps where there is little to add: the SM adds two doubles a clock)
    const int warps = min(kThreads / 32, (g.chunks + 63) / 64);
    __shared__ double sums[kThreads / 32];
    if ((int)threadIdx.x < 32 * warps) {
        double sum = 0.0;
        for (int i = threadIdx.x; i < g.chunks; i += 32 * warps)
            sum += g.partial[(int64_t)matrix * g.chunks + i];
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
        if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = sum;
        if (warps > 1)
            asm volatile("bar.sync 1, %0;" ::"r"(32 * warps) : "memory");
        if (threadIdx.x == 0) {
            for (int w = 1; w < warps; ++w) sum += sums[w];
            const bool usual = sum > 1e-30 && sum < 1e30 && args.eps < 1e30;
            s_f = usual ? kOrthoScale / (sqrtf((float)sum) + (float)args.eps) : 0.f;
            if (!usual) s_factor = (double)kOrthoScale / (sqrt(sum) + args.eps);
        }
    }
    __syncthreads();
    const float f = s_f;
    const auto scaled = [&](float u) { return f > 0.f ? u * f : (float)((double)u * s_factor); };

    const int64_t base = (int64_t)matrix * g.m * g.ldx;
    const auto store = [&](int r, int c, const float (&v)[4]) {  // columns c .. c + 3 of X
        if (r >= g.m || c >= g.n) return;
        const uint32_t h0 = pack(v[0], v[1]), h1 = pack(v[2], v[3]);
        const float2 a = unpack(h0), z = unpack(h1);
        *reinterpret_cast<uint2 *>(g.x[0] + base + (int64_t)r * g.ldx + c) = make_uint2(h0, h1);
        uint4 *rest = g.rest + ((int64_t)(matrix * g.blocks_down + r / 32) * g.blocks_across +
                                c / 32) * kBlockPieces + c % 32 / 8 * 32 + r % 32;
        reinterpret_cast<uint2 *>(rest)[c % 8 / 4] =
            make_uint2(pack(v[0] - a.x, v[1] - a.y), pack(v[2] - z.x, v[3] - z.y));
    };
    if (s.by4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int y = ty + 16 * i, r = r0 + y, c = c0 + tx;
            float v[4] = {in[i].x, in[i].y, in[i].z, in[i].w};
            if (s.momentum) {
                const float o[4] = {old[i].x, old[i].y, old[i].z, old[i].w};
                float n[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    n[j] = s.mo.next(o[j], v[j]);
                    v[j] = s.mo.u(n[j], v[j]);
                }
                if (r < g.rows && c < g.cols)
                    *reinterpret_cast<float4 *>(s.momentum + s.at + r * s.stride + c) =
                        make_float4(n[0], n[1], n[2], n[3]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = scaled(v[j]);
            if (!g.tall) {
                store(r, c, v);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) tile[y][tx + j] = v[j];
            }
        }
        if (!g.tall) return;
    } else {
#pragma unroll 4
        for (int i = threadIdx.x; i < kPrep * kPrep; i += kThreads) {
            const int y = i / kPrep, x = i % kPrep, r = r0 + y, c = c0 + x;
            float u = 0.f;
            if (r < g.rows && c < g.cols) {
                const int64_t e = s.at + r * s.stride + c;
                u = param_load(s.in, e, s.bf16);
                if (s.momentum) {
                    const float b1 = s.mo.next(s.momentum[e], u);
                    s.momentum[e] = b1;
                    u = s.mo.u(b1, u);
                }
            }
            tile[y][x] = scaled(u);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int y = ty + 16 * i;
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = g.tall ? tile[tx + j][y] : tile[y][tx + j];
        store((g.tall ? c0 : r0) + y, (g.tall ? r0 : c0) + tx, v);
    }
}

template <typename K>
cudaError_t launch(K kernel, const OrthoArgs &a, int grid, int threads, int ctas, int smem,
                   cudaStream_t stream) {
    if (grid == 0) return cudaSuccess;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(grid);
    c.blockDim = dim3(threads);
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

template <int kCtas, bool kOutBf16, bool kParts>
cudaError_t launch_chain(const OrthoArgs &a, int sm_count, cudaStream_t stream) {
    static PerDevice ready;
    const auto kernel = ortho_chain_kernel<kCtas, kOutBf16, kParts>;
    const int d = PerDevice::device();
    if (!ready.get(d)) {
        const cudaError_t e = cudaFuncSetAttribute(
            kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes);
        if (e != cudaSuccess) return e;
        ready.set(d, 1);
    }
    const int most = sm_count / kCtas;
    return launch(kernel, a, (a.tiles < most ? a.tiles : most) * kCtas, kProductThreads, kCtas,
                  kSharedBytes, stream);
}

}  // namespace

int ortho_pair_tile() { return 2 * kHalfTile; }
int ortho_slot_depth() { return kK; }
int ortho_epilogue_warps() { return kEpilogueWarps; }

cudaError_t launch_ortho_norm(const OrthoArgs &a, cudaStream_t stream) {
    return launch(ortho_norm_kernel, a, a.norm_blocks, kThreads, 1, 0, stream);
}

cudaError_t launch_ortho_prepare(const OrthoArgs &a, cudaStream_t stream) {
    return launch(ortho_prepare_kernel, a, a.prep_blocks, kThreads, 1, 0, stream);
}

cudaError_t launch_ortho_chain(const OrthoArgs &a, int ctas, int sm_count, cudaStream_t stream) {
    bool parts = false;
    for (int i = 0; i < a.n_groups; ++i)
        parts = parts || a.g[i].split[0] > 1 || a.g[i].split[1] > 1;
    const auto by = [&](auto n, auto p) {
        return a.out_bf16 ? launch_chain<n.value, true, p.value>(a, sm_count, stream)
                          : launch_chain<n.value, false, p.value>(a, sm_count, stream);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    if (ctas == 1) return parts ? by(one, std::true_type()) : by(one, std::false_type());
    return parts ? by(two, std::true_type()) : by(two, std::false_type());
}

}  // namespace aloco
