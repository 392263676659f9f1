// Entry points of the orthogonalised updates: argument checks, the split of
// the matrices into passes, and the passes' launches (aloco_orthogonal.cu).
#include <algorithm>
#include <array>
#include <cmath>
#include <limits>
#include <new>
#include <vector>

#include "aloco_checks.h"
#include "aloco_orthogonal.h"

// The testing hook of aloco_test_stall_tile (aloco_host.cpp).
extern thread_local int64_t t_test_stall_tile1;

using namespace aloco;

namespace {

// Scratch that a pass may fill.  More matrices at once fill the tiles' last
// round better; a pass of this size holds thousands of tiles.
constexpr size_t kPassBytes = (size_t)3 << 30;
constexpr size_t kAlign = 256;

size_t up(size_t x, size_t to) { return (x + to - 1) / to * to; }

// SMs that passes are planned for: scratch is reckoned without a device.
constexpr int kPlannedSms = 152;

// Matrices of one shape: `period` places of M workers.
struct Shape {
    int64_t rows, cols;
    int first, period;               // places [first, first + period)
    bool merged;                     // may take two steps at a time
    int64_t chunk;                   // elements of a norm block
    int64_t m() const { return std::min(rows, cols); }
    int64_t n() const { return std::max(rows, cols); }
    int64_t ldx() const { return (int64_t)up((size_t)n(), 8); }
    int64_t lda() const { return (int64_t)up((size_t)m(), 8); }
    int64_t chunks() const { return (rows * cols + chunk - 1) / chunk; }
    // places for symmetric matrices
    int syms() const { return merged ? kOrthoSyms : 2; }
    int64_t down() const { return (m() + 31) / 32; }
    int64_t across() const { return (n() + 31) / 32; }
    size_t rest_bytes() const { return (size_t)(down() * across()) * 2048; }
    // scratch of `count` matrices
    size_t bytes(int64_t count) const {
        return 2 * up((size_t)(count * m() * ldx()) * 2, kAlign) + (size_t)count * rest_bytes() +
               syms() * (up((size_t)(count * m() * lda()) * 2, kAlign) +
                         up((size_t)(count * m()) * 4, kAlign)) +
               up((size_t)(count * chunks()) * 8, kAlign);
    }
};

int64_t tiles_of(int64_t x, int tile) { return (x + tile - 1) / tile; }
int64_t sym_tiles(const Shape &s, int tile) {
    const int64_t rows = tiles_of(s.m(), tile);
    return rows * (rows + 1) / 2;
}

// A part of a shape's matrices: those from `skip` on.
struct Part {
    int shape;
    int64_t skip, count;
};
// Matrices that go through the products' kernel together.
struct Pass {
    std::vector<Part> parts;
    int places = 0;
    size_t bytes = 0;                // but for what follows from the tiles:
    int ctas = 2;                    // that share one
    std::vector<std::array<int, 2>> split;  // by part: of A's and P's tiles
    size_t counters = 0;             // ints that begin as zero
    size_t all_bytes = 0;
};

// Matrices that one kernel takes through all steps, `ctas` to a matrix.
struct SmallPass {
    int ctas;
    std::vector<Part> parts;
    int places = 0;
};

struct Plan {
    std::vector<int64_t> place;
    std::vector<Shape> shapes;
    std::vector<Pass> passes;
    std::vector<SmallPass> small;
    size_t bytes = 0;
};

// CTAs of a small matrix, a power of two; 0: it is none.
int small_ctas(const Shape &s, int most) {
    if (s.m() > kOrthoSmallSide) return 0;
    for (int c = 1; c <= most; c *= 2)
        if (s.n() <= (int64_t)c * kOrthoSmallCols) return c;
    return 0;
}

// The largest cluster that every device takes, which scratch is reckoned with.
constexpr int kPortableCtas = 8;

// Bytes of the sums that the parts of a group's tiles leave.
size_t sums_bytes(const Shape &s, int64_t count, const std::array<int, 2> &split, int tile) {
    const int parts = std::max(split[0], split[1]);
    return parts > 1 ? (size_t)(count * sym_tiles(s, tile) * parts) * tile * tile * 4 : 0;
}

// Tiles by pairs of CTAs where the matrices' elements fill them; by single CTAs, whose
// tiles are a quarter, below: 8 matrices of 300 x 2000 192 us by single ones and 225 by
// pairs, 7 odd ones of 3 workers 217 and 254, where a matrix's edges count as whole
// tiles too; 3 of 1500 x 1500 (103 tiles' elements) 333 and 302.  Where A's or P's tiles
// are fewer than the CTAs, parts of their depth are tiles of their own: as many as there
// are CTAs for, of at least 12 slots.  (5632 x 2048 alone: 88 slots a tile of A, 36 tiles
// for 76 pairs.)
void lay_out(const Plan &plan, Pass *pass) {
    int64_t elements = 0;
    for (const Part &part : pass->parts) {
        const Shape &s = plan.shapes[part.shape];
        elements += part.count * s.m() * s.n();
    }
    const int64_t tile_elements = (int64_t)ortho_pair_tile() * ortho_pair_tile();
    pass->ctas = elements >= kPlannedSms / 2 * tile_elements ? 2 : 1;
    const int tile = ortho_pair_tile() / 2 * pass->ctas, slots = kPlannedSms / pass->ctas;
    pass->split.assign(pass->parts.size(), {1, 1});
    for (int what = 0; what < 2; ++what) {
        const auto chunks = [&](const Part &part) {
            const Shape &s = plan.shapes[part.shape];
            return tiles_of(what == 0 ? s.n() : s.m(), ortho_slot_depth());
        };
        int64_t most = 0, tiles = 0;
        for (const Part &part : pass->parts) {
            most = std::max(most, chunks(part));
            tiles += part.count * sym_tiles(plan.shapes[part.shape], tile);
        }
        if (tiles >= slots) continue;
        for (int64_t depth = 12; depth < most; depth = depth * 5 / 4) {
            int64_t parts = 0;
            for (const Part &part : pass->parts)
                parts += part.count * sym_tiles(plan.shapes[part.shape], tile) *
                         tiles_of(chunks(part), (int)depth);
            if (parts > slots) continue;
            for (size_t i = 0; i < pass->parts.size(); ++i)
                pass->split[i][what] = (int)tiles_of(chunks(pass->parts[i]), (int)depth);
            break;
        }
    }
    pass->counters = kOrthoCounters;
    pass->all_bytes = pass->bytes;
    for (size_t i = 0; i < pass->parts.size(); ++i) {
        const Part &part = pass->parts[i];
        const Shape &s = plan.shapes[part.shape];
        pass->counters += (size_t)part.count;
        const size_t sums = sums_bytes(s, part.count, pass->split[i], tile);
        if (!sums) continue;
        pass->counters += (size_t)(part.count * sym_tiles(s, tile)) * pass->ctas *
                          ortho_epilogue_warps() * 2;
        pass->all_bytes += up(sums, kAlign);
    }
    pass->all_bytes += up(pass->counters * 4, kAlign);
}

// Two steps at a time (list_operations), by the matrix's shape alone: its rounding must
// not depend on what else a call holds.  They save 3 m m (n - m) products of the
// two steps' and add two dependent products of m x m.  One matrix of 512 x 2048 takes
// 188 us with them and 176 without, 1024 x 2048 244 and 232, 1500 x 2250 307 and 326,
// 2048 x 8192 543 and 656; 64 of 512 x 2048 757 and 933, of 768 x 1536 1064 and 1235,
// of 1024 x 1536 1711 and 1885.  Below the limit they are left out, although many of 512
// x 1024 (64: 497 and 543) would gain: one alone loses (179 and 163).
bool two_at_a_time(int64_t m, int64_t n) {
    return 2 * n >= 3 * m && m * m * (n - m) >= (int64_t)1 << 28;
}

// Shapes in `p` (places set) into passes that keep within kPassBytes, kOrthoGroups
// and kOrthoMatrices: deep products first, so that the last tiles are short.
// Where all are small they go through the small kernel, in clusters of up to
// `most_ctas`.
void split(Plan *p, int workers, int most_ctas) {
    std::stable_sort(p->shapes.begin(), p->shapes.end(), [](const Shape &x, const Shape &y) {
        return x.m() != y.m() ? x.m() > y.m() : x.n() > y.n();
    });
    // Norm blocks: two rounds of eight an SM, of 4096 to 65536 elements; at most 1024 of
    // a matrix.
    for (Shape &s : p->shapes) {
        const int64_t all = s.period * (int64_t)workers, size = s.rows * s.cols;
        s.merged = two_at_a_time(s.m(), s.n());
        const int64_t each = std::min<int64_t>(65536, all * size / (kPlannedSms * 16));
        s.chunk = std::max<int64_t>(4096, (int64_t)up((size_t)std::max(each, size / 1024), 4096));
    }
    // (beside larger ones the small fill tiles of the kernels that run anyway)
    bool all = true;
    for (const Shape &s : p->shapes) all = all && small_ctas(s, most_ctas);
    std::vector<SmallPass> open;     // by cluster size
    for (int i = 0; all && i < (int)p->shapes.size(); ++i) {
        const Shape &s = p->shapes[i];
        const int ctas = small_ctas(s, most_ctas);
        auto at = std::find_if(open.begin(), open.end(),
                               [&](const SmallPass &x) { return x.ctas == ctas; });
        if (at != open.end() &&
            (at->parts.size() == kOrthoGroups || at->places + s.period > kOrthoMatrices)) {
            p->small.push_back(std::move(*at));
            open.erase(at);
            at = open.end();
        }
        if (at == open.end()) {
            open.push_back({ctas, {}, 0});
            at = open.end() - 1;
        }
        at->parts.push_back({i, 0, (int64_t)s.period * workers});
        at->places += s.period;
    }
    for (SmallPass &x : open) p->small.push_back(std::move(x));

    Pass pass;
    const auto flush = [&] {
        if (pass.parts.empty()) return;
        lay_out(*p, &pass);
        p->bytes = std::max(p->bytes, pass.all_bytes);
        p->passes.push_back(std::move(pass));
        pass = Pass();
    };
    for (int i = 0; !all && i < (int)p->shapes.size(); ++i) {
        const Shape &s = p->shapes[i];
        const int64_t total = (int64_t)s.period * workers;
        for (int64_t at = 0; at < total;) {
            if (pass.parts.size() == kOrthoGroups || pass.places + s.period > kOrthoMatrices)
                flush();
            const size_t room = kPassBytes - std::min(kPassBytes, pass.bytes);
            int64_t fit = (int64_t)(room / s.bytes(1));
            if (fit == 0 && !pass.parts.empty()) {
                flush();
                continue;
            }
            fit = std::max<int64_t>(fit, 1);
            // equal parts where one does not hold all
            const int64_t left = total - at, parts = (left + fit - 1) / fit;
            const int64_t count = pass.parts.empty() ? (left + parts - 1) / parts
                                                     : std::min(left, fit);
            pass.parts.push_back({i, at, count});
            pass.places += s.period;
            pass.bytes += s.bytes(count);
            at += count;
        }
    }
    flush();
}

// Matrices by shape, in the order of their places.
void plan_matrices(const aloco_matrix_t *mats, int64_t n, int workers, int most_ctas, Plan *p) {
    std::vector<int64_t> order;
    for (int64_t i = 0; i < n; ++i)
        if (mats[i].rows > 0 && mats[i].cols > 0) order.push_back(i);
    std::stable_sort(order.begin(), order.end(), [&](int64_t a, int64_t b) {
        const aloco_matrix_t &x = mats[a], &y = mats[b];
        return x.rows != y.rows ? x.rows < y.rows : x.cols < y.cols;
    });
    for (const int64_t i : order) {
        const aloco_matrix_t &x = mats[i];
        if (p->shapes.empty() || p->shapes.back().rows != x.rows ||
            p->shapes.back().cols != x.cols || p->shapes.back().period == 256)
            p->shapes.push_back({x.rows, x.cols, (int)p->place.size(), 0, false, 0});
        ++p->shapes.back().period;
        p->place.push_back(x.offset);
    }
    split(p, workers, most_ctas);
}

void plan_batch(int64_t batch, int64_t rows, int64_t cols, int most_ctas, Plan *p) {
    for (int64_t i = 0; i < batch; ++i) {
        if (p->shapes.empty() || p->shapes.back().period == 256)
            p->shapes.push_back({rows, cols, (int)i, 0, false, 0});
        ++p->shapes.back().period;
        p->place.push_back(i);
    }
    split(p, 1, most_ctas);
}

int check_side(int64_t rows, int64_t cols, const char *what, int64_t i) {
    if (rows < 0 || cols < 0 || std::min(rows, cols) > ALOCO_MAX_SIDE ||
        std::max(rows, cols) > ALOCO_MAX_LONG_SIDE)
        return fail(ALOCO_ERR_ARG, "%s[%lld]: %lld x %lld out of range (sides up to %d and %d)",
                    what, (long long)i, (long long)rows, (long long)cols, ALOCO_MAX_SIDE,
                    ALOCO_MAX_LONG_SIDE);
    return ALOCO_OK;
}

int check_steps(const double (*coefficients)[3], int32_t steps, double eps) {
    if (steps < 1 || steps > ALOCO_MAX_NS_STEPS)
        return fail(ALOCO_ERR_ARG, "steps = %d outside [1, %d]", steps, ALOCO_MAX_NS_STEPS);
    for (int s = 0; s < steps; ++s)
        for (int i = 0; i < 3; ++i)
            if (!(std::fabs(coefficients[s][i]) <= 100.0))
                return fail(ALOCO_ERR_ARG, "coefficients[%d][%d] = %g outside [-100, 100]", s, i,
                            coefficients[s][i]);
    if (!(std::isfinite(eps) && eps >= 1e-30))
        return fail(ALOCO_ERR_ARG, "eps = %g must be finite and >= 1e-30", eps);
    return ALOCO_OK;
}

// A map of `count` matrices of rows x cols fp16 values, ld elements a row, in
// boxes of 64 x 64.
int tensor_map(CUtensorMap *map, void *data, int64_t cols, int64_t rows, int64_t ld,
               int64_t count) {
    typedef CUresult (*Fn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                           const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                           const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                           CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Fn fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000,
                                             cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return (Fn)f;
    }();
    if (!fn) return fail(ALOCO_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)count};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)(ld * rows) * 2};
    const cuuint32_t box[3] = {64, 64, 1}, step[3] = {1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, data, dims, strides, box, step,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(ALOCO_ERR_CUDA, "cuTensorMapEncodeTiled: error %d (%lld x %lld x %lld)",
                    (int)r, (long long)cols, (long long)rows, (long long)count);
    return ALOCO_OK;
}

// What both kinds of passes fill in of a group.
void fill_group(const Plan &plan, const Part &part, int64_t *places, int *n_places,
                OrthoGroup *g) {
    const Shape &s = plan.shapes[part.shape];
    *g = OrthoGroup();
    g->m = (int)s.m();
    g->n = (int)s.n();
    g->rows = (int)s.rows;
    g->cols = (int)s.cols;
    g->tall = s.rows > s.cols;
    g->count = (int)part.count;
    g->first = *n_places;
    g->period = s.period;
    g->skip = (int)part.skip;
    for (int k = 0; k < s.period; ++k) places[(*n_places)++] = plan.place[s.first + k];
}

int run_small(const Plan &plan, const SmallPass &pass, const OrthoArgs &base,
              const double *shape_step, cudaStream_t stream) {
    OrthoArgs a = base;
    a.n_groups = (int)pass.parts.size();
    a.small_ctas = pass.ctas;
    int places = 0, matrices = 0;
    for (int i = 0; i < a.n_groups; ++i) {
        fill_group(plan, pass.parts[i], a.place, &places, &a.g[i]);
        a.g[i].small0 = matrices;
        matrices += a.g[i].count;
        a.step[i] = shape_step ? (float)shape_step[pass.parts[i].shape] : 0.f;
    }
    const cudaError_t e = launch_ortho_small(a, matrices, stream);
    return e == cudaSuccess ? ALOCO_OK : cuda_fail(e, "orthogonal factor");
}

// `base`: the caller's buffers and settings filled in.
int run_pass(const Plan &plan, const Pass &pass, const OrthoArgs &base, const double *shape_step,
             char *scratch, int sm_count, cudaStream_t stream) {
    OrthoArgs a = base;
    char *at = scratch;
    const auto take = [&](size_t bytes) {
        char *p = at;
        at += up(bytes, kAlign);
        return p;
    };
    a.n_groups = (int)pass.parts.size();
    int places = 0, norm = 0, prep = 0;
    a.counters = (int)pass.counters;
    a.next_tile = (int *)take(pass.counters * 4);
    int *counter = a.next_tile + kOrthoCounters;
    const int tile = ortho_pair_tile() / 2 * pass.ctas;
    for (int i = 0; i < a.n_groups; ++i) {
        const Part &part = pass.parts[i];
        const Shape &s = plan.shapes[part.shape];
        OrthoGroup &g = a.g[i];
        const int64_t m = s.m(), n = s.n(), count = part.count;
        fill_group(plan, part, a.place, &places, &g);
        g.ldx = (int)s.ldx();
        g.lda = (int)s.lda();
        g.chunk = (int)s.chunk;
        g.chunks = (int)s.chunks();
        g.norm0 = norm;
        norm += g.chunks * g.count;
        g.prep0 = prep;
        prep += (int)((s.rows + 63) / 64 * ((s.cols + 63) / 64)) * g.count;
        const size_t x_bytes = (size_t)(count * m * s.ldx()) * 2;
        const size_t a_bytes = (size_t)(count * m * s.lda()) * 2;
        for (int k = 0; k < 2; ++k) g.x[k] = (__half *)take(x_bytes);
        g.rest = (uint4 *)take((size_t)count * s.rest_bytes());
        g.blocks_down = (int)s.down();
        g.blocks_across = (int)s.across();
        g.list = s.merged && base.n_ops[kMerged] ? kMerged : kPlain;
        for (int k = 0; k < s.syms(); ++k) {
            g.sym[k] = (__half *)take(a_bytes);
            g.diag[k] = (float *)take((size_t)(count * m) * 4);
        }
        g.partial = (double *)take((size_t)(count * s.chunks()) * 8);
        g.done = counter;
        counter += count;
        g.sym_tiles = (int)sym_tiles(s, tile);
        g.up_tiles = (int)(tiles_of(m, tile) * tiles_of(n, tile));
        for (int k = 0; k < 2; ++k) g.split[k] = pass.split[i][k];
        for (int k = 0; k < base.n_ops[g.list]; ++k) {
            const OrthoOp &op = base.ops[g.list][k];
            a.tiles += g.count * (op.what == kUpdate ? g.up_tiles
                                                     : g.sym_tiles * g.split[op.what != kGram]);
        }
        if (const size_t sums = sums_bytes(s, count, pass.split[i], tile)) {
            g.sums = (float4 *)take(sums);
            g.came = counter;
            counter += count * g.sym_tiles * pass.ctas * ortho_epilogue_warps() * 2;
        }
        a.step[i] = shape_step ? (float)shape_step[part.shape] : 0.f;
        int rc;
        for (int k = 0; k < 2; ++k)
            if ((rc = tensor_map(&a.map[kMapX0 + k][i], g.x[k], n, m, s.ldx(), count)) != ALOCO_OK)
                return rc;
        for (int k = 0; k < s.syms(); ++k)
            if ((rc = tensor_map(&a.map[kMapSym + k][i], g.sym[k], m, m, s.lda(), count)) !=
                ALOCO_OK)
                return rc;
    }
    a.norm_blocks = norm;
    a.prep_blocks = prep;
    cudaError_t e = launch_ortho_norm(a, stream);
    if (e == cudaSuccess) e = launch_ortho_prepare(a, stream);
    if (e == cudaSuccess) e = launch_ortho_chain(a, pass.ctas, sm_count, stream);
    return e == cudaSuccess ? ALOCO_OK : cuda_fail(e, "orthogonal factor");
}

// The lists of operations.  One step: A = X X^T, P = a + b A + c A A, X <- P X.  Two,
// of m x m matrices but for the first and last product:
//   A = X X^T,  P = p(A),  A' = P A P  (which is X' X'^T),  X <- p'(A') P X
// of which all factors commute, so that every product is symmetric: 3 n + 5 m
// products of m^2 in place of 6 n + 2 m (halved where symmetric).  The factor's
// error is up to three times as large, so only for results in bf16.
void list_operations(const double (*coefficients)[3], int steps, bool bf16, OrthoArgs *a) {
    const auto add = [&](int list, OrthoOp op) {
        int &n = a->n_ops[list];
        if (n) {
            const OrthoOp &last = a->ops[list][n - 1];
            op.syms = (int8_t)(last.syms + (last.what != kUpdate));
            op.ups = (int8_t)(last.ups + (last.what == kUpdate));
        }
        a->ops[list][n++] = op;
    };
    const auto op = [](int what, int left, int right, int out, int step, int x) {
        OrthoOp o{};
        o.what = (int8_t)what;
        o.left = (int8_t)left;
        o.right = (int8_t)right;
        o.out = (int8_t)out;
        o.step = (int8_t)step;
        o.x = (int8_t)x;
        return o;
    };
    const auto one = [&](int list, int s, int x) {
        // (where e = b / 2c is not large against A)
        const float b = (float)coefficients[s][1], c = (float)coefficients[s][2];
        const bool shifted = c != 0.f && std::fabs(b) <= 4 * std::fabs(c);
        OrthoOp o = op(kGram, 0, 0, 0, s, x);
        o.shifted = shifted;
        add(list, o);
        o = op(kPoly, 0, 0, 1, s, x);
        o.shifted = shifted;
        o.bare = 1;
        add(list, o);
        o = op(kUpdate, 1, 0, 0, s, x);
        o.last = s + 1 == steps;
        add(list, o);
    };
    for (int s = 0; s < steps; ++s) one(kPlain, s, s & 1);
    if (!bf16 || steps < 2) return;
    int x = 0;
    for (int s = 0; s < steps; s += 2, x ^= 1) {
        if (s + 1 == steps) {
            one(kMerged, s, x);
            break;
        }
        add(kMerged, op(kGram, 0, 0, 0, s, x));
        add(kMerged, op(kPoly, 0, 0, 1, s, x));
        add(kMerged, op(kProduct, 1, 0, 2, s, x));
        add(kMerged, op(kProduct, 2, 1, 0, s, x));
        add(kMerged, op(kPoly, 0, 0, 3, s + 1, x));
        OrthoOp o = op(kProduct, 3, 1, 2, s, x);
        o.bare = 1;
        add(kMerged, o);
        o = op(kUpdate, 2, 0, 0, s, x);
        o.last = s + 2 == steps;
        add(kMerged, o);
    }
}

// All of a call's passes.
int run(const Plan &plan, const OrthoArgs &base, const double (*coefficients)[3], int steps,
        const double *shape_step, char *scratch, int sm_count, cudaStream_t stream) {
    OrthoArgs a = base;
    a.steps = steps;
    for (int s = 0; s < steps; ++s)
        for (int i = 0; i < 3; ++i) a.coef[s][i] = (float)coefficients[s][i];
    list_operations(coefficients, steps, a.out_bf16, &a);
    for (const SmallPass &pass : plan.small) {
        const int rc = run_small(plan, pass, a, shape_step, stream);
        if (rc != ALOCO_OK) return rc;
        a.test_stall1 = 0;
    }
    for (const Pass &pass : plan.passes) {
        const int rc = run_pass(plan, pass, a, shape_step, scratch, sm_count, stream);
        if (rc != ALOCO_OK) return rc;
        a.test_stall1 = 0;
    }
    return done();
}

// The plan that the device takes: with its largest clusters, unless that would
// want more scratch than callers were told of.
template <typename F>
int device_plan(const F &make, Plan *plan) {
    bool fits = false, larger = false;
    cudaError_t e = cudaSuccess;
    for (const SmallPass &s : plan->small) {
        if ((e = ortho_small_setup(s.ctas, &fits)) != cudaSuccess) break;
        if (!fits)
            return fail(ALOCO_ERR_CUDA, "the device has no room for a cluster of %d", s.ctas);
    }
    for (const Shape &s : plan->shapes)
        larger = larger || small_ctas(s, kOrthoSmallCtas) > kPortableCtas;
    for (const Shape &s : plan->shapes) larger = larger && small_ctas(s, kOrthoSmallCtas);
    if (e == cudaSuccess && larger) e = ortho_small_setup(kOrthoSmallCtas, &fits);
    if (e != cudaSuccess) return cuda_fail(e, "orthogonal factor");
    if (larger && fits) {
        Plan other;
        make(kOrthoSmallCtas, &other);
        for (const SmallPass &s : other.small)
            if ((e = ortho_small_setup(s.ctas, &fits)) != cudaSuccess)
                return cuda_fail(e, "orthogonal factor");
        if (other.bytes <= plan->bytes) *plan = std::move(other);
    }
    return ALOCO_OK;
}

int check_scratch(const void *scratch, size_t bytes, size_t need) {
    if (need == 0) return ALOCO_OK;
    if (bytes < need)
        return fail(ALOCO_ERR_ARG, "scratch of %zu bytes, need %zu", bytes, need);
    if (!scratch) return fail(ALOCO_ERR_ARG, "NULL scratch");
    if ((uintptr_t)scratch & (kAlign - 1))
        return fail(ALOCO_ERR_ARG, "scratch: not aligned to %zu bytes", kAlign);
    return ALOCO_OK;
}

bool meet(const void *p, size_t m, const void *q, size_t n) {
    return (uintptr_t)p < (uintptr_t)q + n && (uintptr_t)q < (uintptr_t)p + m;
}

// (a copy that comes late is asked of other calls: it stays for them)
int64_t take_stall() {
    const int64_t s = t_test_stall_tile1;
    if (s <= 0) return 0;
    t_test_stall_tile1 = 0;
    return s;
}

// The matrices lie in a vector of N elements (N < 0: any) and do not overlap.
int check_matrices(const aloco_matrix_t *mats, int64_t n, int64_t N) {
    if (n < 0 || n > (1 << 20)) return fail(ALOCO_ERR_ARG, "n = %lld out of range", (long long)n);
    if (n > 0 && !mats) return fail(ALOCO_ERR_ARG, "NULL matrices");
    std::vector<std::pair<int64_t, int64_t>> spans;
    bool sorted = true;
    for (int64_t i = 0; i < n; ++i) {
        const aloco_matrix_t &x = mats[i];
        const int rc = check_side(x.rows, x.cols, "matrices", i);
        if (rc != ALOCO_OK) return rc;
        const int64_t size = x.rows * x.cols;
        if (x.offset < 0 || x.offset > std::numeric_limits<int64_t>::max() / 8 ||
            (N >= 0 && (x.offset > N || size > N - x.offset)))
            return fail(ALOCO_ERR_ARG, "matrices[%lld]: %lld x %lld from %lld does not lie in a "
                        "vector of %lld", (long long)i, (long long)x.rows, (long long)x.cols,
                        (long long)x.offset, (long long)N);
        if (!size) continue;
        sorted = sorted && (spans.empty() || spans.back().first <= x.offset);
        spans.push_back({x.offset, x.offset + size});
    }
    if (!sorted) std::sort(spans.begin(), spans.end());
    for (size_t i = 1; i < spans.size(); ++i)
        if (spans[i].first < spans[i - 1].second)
            return fail(ALOCO_ERR_ALIAS, "two matrices overlap at element %lld",
                        (long long)spans[i].first);
    return ALOCO_OK;
}

int muon_step(void *const *params, const void *const *grads, float *const *momentum, size_t N,
              int M, aloco_dtype param_dtype, aloco_dtype grad_dtype, const aloco_matrix_t *mats,
              int64_t n, const aloco_muon_cfg_t *cfg, void *scratch, size_t scratch_bytes,
              const aloco_opts_t *opts) {
    int rc;
    if (!cfg) return fail(ALOCO_ERR_ARG, "NULL cfg");
    if (!params || !grads || !momentum) return fail(ALOCO_ERR_ARG, "NULL buffer array");
    if (M < 1 || M > ALOCO_MAX_WORKERS)
        return fail(ALOCO_ERR_ARG, "M = %d outside [1, %d]", M, ALOCO_MAX_WORKERS);
    if ((param_dtype != ALOCO_F32 && param_dtype != ALOCO_BF16) ||
        (grad_dtype != ALOCO_F32 && grad_dtype != ALOCO_BF16))
        return fail(ALOCO_ERR_ARG, "unknown dtype (params %d, grads %d)", (int)param_dtype,
                    (int)grad_dtype);
    if (N > (size_t)std::numeric_limits<int64_t>::max() / 8)
        return fail(ALOCO_ERR_ARG, "N = %zu out of range", N);
    if (!(std::isfinite(cfg->lr) && cfg->lr >= 0.0))
        return fail(ALOCO_ERR_ARG, "lr = %g must be finite and >= 0", cfg->lr);
    if (!(cfg->momentum >= 0.0 && cfg->momentum < 1.0))
        return fail(ALOCO_ERR_ARG, "momentum = %g outside [0, 1)", cfg->momentum);
    if (!(std::isfinite(cfg->weight_decay) && cfg->weight_decay >= 0.0))
        return fail(ALOCO_ERR_ARG, "weight_decay = %g must be finite and >= 0", cfg->weight_decay);
    if (cfg->nesterov != 0 && cfg->nesterov != 1)
        return fail(ALOCO_ERR_ARG, "nesterov = %d must be 0 or 1", cfg->nesterov);
    if (cfg->scale < ALOCO_MUON_ADAMW || cfg->scale > ALOCO_MUON_UNIT)
        return fail(ALOCO_ERR_ARG, "unknown scale %d", cfg->scale);
    if ((rc = check_steps(cfg->coefficients, cfg->steps, cfg->eps)) != ALOCO_OK) return rc;
    if ((rc = check_matrices(mats, n, (int64_t)N)) != ALOCO_OK) return rc;
    Plan plan;
    const auto make = [&](int ctas, Plan *p) { plan_matrices(mats, n, M, ctas, p); };
    make(kPortableCtas, &plan);
    if (plan.passes.empty() && plan.small.empty()) return done();
    if ((rc = check_scratch(scratch, scratch_bytes, plan.bytes)) != ALOCO_OK) return rc;

    const size_t px = param_dtype == ALOCO_F32 ? 4 : 2, pg = grad_dtype == ALOCO_F32 ? 4 : 2;
    struct Buf { const void *p; size_t bytes, size; bool written; const char *name; int i; };
    Buf bufs[3 * ALOCO_MAX_WORKERS + 1];
    int nb = 0;
    for (int i = 0; i < M; ++i) {
        bufs[nb++] = {params[i], N * px, px, true, "params", i};
        bufs[nb++] = {grads[i], N * pg, pg, false, "grads", i};
        bufs[nb++] = {momentum[i], N * 4, 4, true, "momentum", i};
    }
    for (int i = 0; i < nb; ++i) {
        if (!bufs[i].p) return fail(ALOCO_ERR_ARG, "NULL %s[%d]", bufs[i].name, bufs[i].i);
        if ((uintptr_t)bufs[i].p & (bufs[i].size - 1))
            return fail(ALOCO_ERR_ARG, "%s[%d]: not aligned to its element", bufs[i].name,
                        bufs[i].i);
    }
    if (plan.bytes) bufs[nb++] = {scratch, plan.bytes, 1, true, "scratch", 0};
    for (int i = 0; i < nb; ++i)
        for (int j = 0; j < i; ++j)
            if ((bufs[i].written || bufs[j].written) &&
                meet(bufs[i].p, bufs[i].bytes, bufs[j].p, bufs[j].bytes))
                return fail(ALOCO_ERR_ALIAS, "%s[%d] and %s[%d] overlap", bufs[j].name, bufs[j].i,
                            bufs[i].name, bufs[i].i);
    int device, sms;
    if ((rc = current_device(&device, &sms)) != ALOCO_OK) return rc;
    RangeCheck check;
    for (int i = 0; i < nb; ++i)
        if ((rc = check(bufs[i].p, bufs[i].bytes, device, bufs[i].name, bufs[i].i)) != ALOCO_OK)
            return rc;

    if ((rc = device_plan(make, &plan)) != ALOCO_OK) return rc;

    OrthoArgs a;
    std::memset(&a, 0, sizeof a);
    a.source = kSourceMuon;
    a.in_bf16 = grad_dtype == ALOCO_BF16;
    a.out_bf16 = param_dtype == ALOCO_BF16;
    for (int i = 0; i < M; ++i) {
        a.in[i] = grads[i];
        a.momentum[i] = momentum[i];
        a.out[i] = params[i];
    }
    a.mu = (float)cfg->momentum;
    a.nesterov = cfg->nesterov;
    a.decay = (float)(1.0 - cfg->lr * cfg->weight_decay);
    a.eps = cfg->eps;
    a.test_stall1 = take_stall();
    std::vector<double> step;
    for (const Shape &s : plan.shapes) {
        const double by = cfg->scale == ALOCO_MUON_ADAMW ? 0.2 * std::sqrt((double)s.n())
                          : cfg->scale == ALOCO_MUON_ASPECT
                              ? std::sqrt(std::max(1.0, (double)s.rows / (double)s.cols))
                              : 1.0;
        step.push_back(-cfg->lr * by);
    }
    return run(plan, a, cfg->coefficients, cfg->steps, step.data(), (char *)scratch, sms,
               stream_of(opts));
}

int orthogonalize(const void *x, int64_t batch, int64_t rows, int64_t cols, int64_t batch_stride,
                  int64_t row_stride, aloco_dtype dtype, void *out, const double *coefficients,
                  int32_t steps, double eps, void *scratch, size_t scratch_bytes,
                  const aloco_opts_t *opts) {
    int rc;
    if (dtype != ALOCO_F32 && dtype != ALOCO_BF16)
        return fail(ALOCO_ERR_ARG, "unknown dtype %d", (int)dtype);
    if (batch < 0 || batch > (1 << 20))
        return fail(ALOCO_ERR_ARG, "batch = %lld out of range", (long long)batch);
    if ((rc = check_side(rows, cols, "x", 0)) != ALOCO_OK) return rc;
    if (!coefficients) return fail(ALOCO_ERR_ARG, "NULL coefficients");
    double steps_of[ALOCO_MAX_NS_STEPS][3];
    if (steps >= 1 && steps <= ALOCO_MAX_NS_STEPS)
        std::memcpy(steps_of, coefficients, sizeof(double) * 3 * (size_t)steps);
    if ((rc = check_steps(steps_of, steps, eps)) != ALOCO_OK) return rc;
    if (batch == 0 || rows == 0 || cols == 0) return done();
    if (rows == 1) row_stride = 0;
    if (batch == 1) batch_stride = 0;
    // (x is only read: rows and matrices may overlap)
    const int64_t limit = std::numeric_limits<int64_t>::max() / 64;
    if (row_stride < 0 || row_stride > limit / rows || batch_stride < 0 ||
        batch_stride > limit / batch)
        return fail(ALOCO_ERR_ARG, "strides (%lld, %lld) out of range", (long long)batch_stride,
                    (long long)row_stride);
    const int64_t extent = (rows - 1) * row_stride + cols;
    Plan plan;
    const auto make = [&](int ctas, Plan *p) { plan_batch(batch, rows, cols, ctas, p); };
    make(kPortableCtas, &plan);
    if ((rc = check_scratch(scratch, scratch_bytes, plan.bytes)) != ALOCO_OK) return rc;
    const size_t size = dtype == ALOCO_F32 ? 4 : 2;
    Buffers s;
    s.add("x", x, (size_t)((batch - 1) * batch_stride + extent) * size, size, false);
    s.add("out", out, (size_t)(batch * rows * cols) * 2, 2, true);
    s.add("scratch", scratch, plan.bytes, kAlign, true);
    int sms;
    if ((rc = check_buffers(s, false, &sms)) != ALOCO_OK) return rc;

    if ((rc = device_plan(make, &plan)) != ALOCO_OK) return rc;

    OrthoArgs a;
    std::memset(&a, 0, sizeof a);
    a.source = kSourceMatrix;
    a.in_bf16 = dtype == ALOCO_BF16;
    a.out_bf16 = 1;
    a.in[0] = x;
    a.out[0] = out;
    a.batch_stride = batch_stride;
    a.row_stride = row_stride;
    a.eps = eps;
    a.test_stall1 = take_stall();
    return run(plan, a, steps_of, steps, nullptr, (char *)scratch, sms, stream_of(opts));
}

int no_memory() { return fail(ALOCO_ERR_NOMEM, "orthogonal factor: out of host memory"); }

}  // namespace

extern "C" {

void aloco_muon_default_cfg(aloco_muon_cfg_t *cfg) {
    if (!cfg) return;
    std::memset(cfg, 0, sizeof *cfg);
    cfg->lr = 4e-4;
    cfg->momentum = 0.95;
    cfg->weight_decay = 0.1;
    cfg->eps = 1e-7;
    cfg->nesterov = 1;
    cfg->scale = ALOCO_MUON_ADAMW;
    cfg->steps = 5;
    for (int s = 0; s < ALOCO_MAX_NS_STEPS; ++s) {
        cfg->coefficients[s][0] = 3.4445;
        cfg->coefficients[s][1] = -4.7750;
        cfg->coefficients[s][2] = 2.0315;
    }
}

size_t aloco_muon_scratch_bytes(const aloco_matrix_t *matrices, int64_t n, int M) {
    try {
        if (M < 1 || M > ALOCO_MAX_WORKERS || check_matrices(matrices, n, -1) != ALOCO_OK)
            return 0;
        Plan plan;
        plan_matrices(matrices, n, M, kPortableCtas, &plan);
        return plan.bytes;
    } catch (const std::bad_alloc &) {
        no_memory();
        return 0;
    }
}

int aloco_muon_step(void *const *params, const void *const *grads, float *const *momentum,
                    size_t N, int M, aloco_dtype param_dtype, aloco_dtype grad_dtype,
                    const aloco_matrix_t *matrices, int64_t n, const aloco_muon_cfg_t *cfg,
                    void *scratch, size_t scratch_bytes, const aloco_opts_t *opts) {
    try {
        return muon_step(params, grads, momentum, N, M, param_dtype, grad_dtype, matrices, n, cfg,
                         scratch, scratch_bytes, opts);
    } catch (const std::bad_alloc &) {
        return no_memory();
    }
}

size_t aloco_orthogonalize_scratch_bytes(int64_t batch, int64_t rows, int64_t cols) {
    try {
        if (batch < 1 || batch > (1 << 20) || rows < 1 || cols < 1 ||
            check_side(rows, cols, "x", 0) != ALOCO_OK)
            return 0;
        Plan plan;
        plan_batch(batch, rows, cols, kPortableCtas, &plan);
        return plan.bytes;
    } catch (const std::bad_alloc &) {
        no_memory();
        return 0;
    }
}

int aloco_orthogonalize(const void *x, int64_t batch, int64_t rows, int64_t cols,
                        int64_t batch_stride, int64_t row_stride, aloco_dtype dtype, void *out,
                        const double *coefficients, int32_t steps, double eps, void *scratch,
                        size_t scratch_bytes, const aloco_opts_t *opts) {
    try {
        return orthogonalize(x, batch, rows, cols, batch_stride, row_stride, dtype, out,
                             coefficients, steps, eps, scratch, scratch_bytes, opts);
    } catch (const std::bad_alloc &) {
        return no_memory();
    }
}

}  // extern "C"
