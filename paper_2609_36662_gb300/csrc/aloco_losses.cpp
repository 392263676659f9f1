// Entry points of the post-training operators: argument checks and launches of
// the losses (aloco_logits.cuh) and of the gradient-list operators
// (aloco_grads.cu).
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <limits>
#include <new>
#include <utility>
#include <vector>

#include "aloco_checks.h"
#include "aloco_grads.h"
#include "aloco_logits.h"
#include "aloco_scores.h"

// The testing hook of aloco_test_stall_tile (aloco_host.cpp).
extern thread_local int64_t t_test_stall_tile1;

using namespace aloco;  // the checks of aloco_checks.h

namespace {

// ----------------------------------------------------------------- losses

// Strides of a [batch, rows, vocab] array, whose rows may not overlap (either
// dimension may be the outer one), and its extent in bytes.
int check_strides(const char *what, int64_t batch, int64_t rows, int64_t vocab,
                  int64_t batch_stride, int64_t row_stride, int64_t size, size_t *bytes) {
    *bytes = 0;
    if (batch == 0 || rows == 0) return ALOCO_OK;
    struct Dim { int64_t n, stride; } in{rows, rows > 1 ? row_stride : 0},
        out{batch, batch > 1 ? batch_stride : 0};
    if (out.n == 1 || (in.n > 1 && in.stride > out.stride)) std::swap(in, out);
    int64_t extent = vocab;
    for (const Dim &d : {in, out}) {
        if (d.n == 1) continue;
        if (d.stride < extent ||
            d.stride > (std::numeric_limits<int64_t>::max() / 32 - extent) / d.n)
            return fail(ALOCO_ERR_ARG, "%s: strides (%lld, %lld) make rows overlap or lie "
                        "out of range", what, (long long)batch_stride, (long long)row_stride);
        extent += (d.n - 1) * d.stride;
    }
    *bytes = (size_t)extent * (size_t)size;
    return ALOCO_OK;
}

// What every loss checks of its tokens; fills the shared arguments and
// buffers.
int take_tokens(const aloco_tokens_t *t, aloco::LogitsArgs *a, Buffers *s) {
    if (!t) return fail(ALOCO_ERR_ARG, "NULL tokens");
    if (t->dtype != ALOCO_F32 && t->dtype != ALOCO_BF16)
        return fail(ALOCO_ERR_ARG, "unknown dtype %d", t->dtype);
    if (t->target_bytes != 4 && t->target_bytes != 8)
        return fail(ALOCO_ERR_ARG, "target_bytes = %d must be 4 or 8", t->target_bytes);
    if (t->vocab < 1 || t->vocab > ALOCO_MAX_VOCAB)
        return fail(ALOCO_ERR_ARG, "vocab = %lld outside [1, %d]", (long long)t->vocab,
                    ALOCO_MAX_VOCAB);
    if (t->batch < 0 || t->rows < 0 ||
        (t->rows > 0 && t->batch > std::numeric_limits<int32_t>::max() / 16 / t->rows))
        return fail(ALOCO_ERR_ARG, "batch = %lld, rows = %lld out of range",
                    (long long)t->batch, (long long)t->rows);
    if (!(std::isfinite(t->temperature) && t->temperature > 0.0) ||
        t->temperature < 1e-6 || t->temperature > 1e6)
        return fail(ALOCO_ERR_ARG, "temperature = %g outside [1e-6, 1e6]", t->temperature);
    const size_t size = t->dtype == ALOCO_F32 ? 4 : 2;
    size_t bytes = 0;
    int rc = check_strides("logits", t->batch, t->rows, t->vocab, t->batch_stride,
                           t->row_stride, (int64_t)size, &bytes);
    if (rc != ALOCO_OK) return rc;
    std::memset(a, 0, sizeof *a);
    a->n = t->batch * t->rows;
    a->vocab = (int)t->vocab;
    a->x = {(char *)t->logits, t->rows, t->batch_stride, t->row_stride};
    a->target = t->targets;
    a->target_bytes = t->target_bytes;
    a->inv_temp = (float)(1.0 / t->temperature);
    // rounded down, so that the rest is positive: -inf times either is -inf
    const double scale = 1.4426950408889634 / t->temperature;
    a->scale = std::nextafterf((float)scale, 0.f);
    a->scale_lo = (float)(scale - (double)a->scale);
    s->add("logits", t->logits, bytes, size, false);
    s->add("targets", t->targets, (size_t)a->n * t->target_bytes, (size_t)t->target_bytes, false);
    return ALOCO_OK;
}

// The same for the scores, from what take_tokens filled in.
void take_scores(const aloco_tokens_t *t, const LogitsArgs &a, int top, ScoresArgs *s) {
    std::memset(s, 0, sizeof *s);
    s->x = a.x;
    s->g = a.g;
    s->n = a.n;
    s->vocab = a.vocab;
    s->bf16 = t->dtype == ALOCO_BF16;
    s->target = a.target;
    s->target_bytes = a.target_bytes;
    const double scale = 1.4426950408889634 / t->temperature;
    s->scale = (float)scale;
    s->tilt = (float)(0.6931471805599453 * (scale / (double)s->scale - 1.0));
    s->inv_temp = a.inv_temp;
    s->top = top;
}

int take_grad(const aloco_tokens_t *t, const aloco_logits_grad_t *g, aloco::LogitsArgs *a,
              Buffers *s, bool *over) {
    *over = false;
    if (!g) return ALOCO_OK;
    const size_t size = t->dtype == ALOCO_F32 ? 4 : 2;
    size_t bytes = 0;
    const int rc = check_strides("grad", t->batch, t->rows, t->vocab, g->batch_stride,
                                 g->row_stride, (int64_t)size, &bytes);
    if (rc != ALOCO_OK) return rc;
    if (a->n > 0 && !g->data) return fail(ALOCO_ERR_ARG, "NULL grad");
    a->g = {(char *)g->data, t->rows, g->batch_stride, g->row_stride};
    *over = g->data == t->logits && (t->batch <= 1 || g->batch_stride == t->batch_stride) &&
            (t->rows <= 1 || g->row_stride == t->row_stride);
    s->add("grad", g->data, bytes, size, true);
    return ALOCO_OK;
}

// Another value for every call: odd times odd, so never 0, and one that memory
// hardly holds by chance.
unsigned long long new_mark() {
    static std::atomic<unsigned long long> calls{0};
    return (2 * calls.fetch_add(1, std::memory_order_relaxed) + 1) * 0x9e3779b97f4a7c15ull;
}

int take_scratch(void *scratch, size_t bytes, aloco::LogitsArgs *a, Buffers *s) {
    const size_t need = aloco_loss_scratch_bytes(a->n);
    if (bytes < need)
        return fail(ALOCO_ERR_ARG, "scratch of %zu bytes, need %zu", bytes, need);
    s->add("scratch", scratch, need, 16, true);
    a->parts = static_cast<aloco::PolicyPart *>(scratch);
    a->stats = reinterpret_cast<float2 *>(a->parts + a->n);
    a->coef = reinterpret_cast<float *>(a->stats + a->n);
    // (of the last 16 bytes, 8 from where 8 divides the address)
    a->claim = reinterpret_cast<unsigned long long *>(
        ((uintptr_t)(a->coef + a->n) + 7) & ~(uintptr_t)7);
    a->ticket = reinterpret_cast<unsigned int *>(a->claim);
    a->mark = new_mark();
    return ALOCO_OK;
}

constexpr int64_t kMostLate = 8000000000;  // cycles, 4 s

void take_stall(aloco::LogitsArgs *a) {
    a->test_stall1 = std::max<int64_t>(t_test_stall_tile1, -kMostLate);
    t_test_stall_tile1 = 0;
}

}  // namespace

extern "C" {

size_t aloco_loss_scratch_bytes(int64_t rows) {
    if (rows <= 0) return 0;
    // a cluster's part, a row's maximum and sum, its coefficient; a ticket or claim
    return (size_t)rows * (sizeof(aloco::PolicyPart) + sizeof(float2) + sizeof(float)) + 16;
}

int aloco_token_logprobs(const aloco_tokens_t *tokens, float *logp, const aloco_opts_t *opts) {
    aloco::LogitsArgs a;
    Buffers s;
    int rc = take_tokens(tokens, &a, &s);
    if (rc != ALOCO_OK) return rc;
    if (a.n == 0) return done();
    s.add("logp", logp, (size_t)a.n * 4, 4, true);
    a.logp = logp;
    int sms;
    if ((rc = check_buffers(s, false, &sms)) != ALOCO_OK) return rc;
    take_stall(&a);
    const cudaError_t e =
        (tokens->dtype == ALOCO_BF16 ? aloco::token_logprobs_bf16 : aloco::token_logprobs_f32)(a, sms, stream_of(opts));
    return e == cudaSuccess ? done() : cuda_fail(e, "token log-probabilities");
}

int aloco_token_scores(const aloco_tokens_t *tokens, int32_t top, float *logp, float *entropy,
                       int32_t *top_ids, float *top_logp, float *stats, const aloco_opts_t *opts) {
    aloco::LogitsArgs a;
    Buffers s;
    int rc = take_tokens(tokens, &a, &s);
    if (rc != ALOCO_OK) return rc;
    if (top < 0 || top > ALOCO_MAX_TOP || top > tokens->vocab)
        return fail(ALOCO_ERR_ARG, "top = %d outside [0, min(vocab, %d)]", top, ALOCO_MAX_TOP);
    if (a.n == 0) return done();
    const size_t each = (size_t)a.n * 4;
    s.add("logp", logp, each, 4, true);
    if (entropy) s.add("entropy", entropy, each, 4, true);
    if (stats) s.add("stats", stats, 2 * each, 8, true);
    s.add("top_ids", top_ids, each * top, 4, true);
    s.add("top_logp", top_logp, each * top, 4, true);
    int sms;
    if ((rc = check_buffers(s, false, &sms)) != ALOCO_OK) return rc;
    aloco::ScoresArgs b;
    take_scores(tokens, a, top, &b);
    b.logp = logp;
    b.entropy = entropy;
    b.stats = reinterpret_cast<float2 *>(stats);
    b.top_ids = top_ids;
    b.top_logp = top_logp;
    const cudaError_t e = aloco::launch_token_scores(b, sms, stream_of(opts));
    return e == cudaSuccess ? done() : cuda_fail(e, "token scores");
}

int aloco_token_scores_grad(const aloco_tokens_t *tokens, const float *stats, const float *entropy,
                            const float *d_logp, const float *d_entropy, int32_t top,
                            const int32_t *top_ids, const float *d_top,
                            const aloco_logits_grad_t *grad, const aloco_opts_t *opts) {
    aloco::LogitsArgs a;
    Buffers s;
    int rc = take_tokens(tokens, &a, &s);
    if (rc != ALOCO_OK) return rc;
    if (top < 0 || top > ALOCO_MAX_TOP)
        return fail(ALOCO_ERR_ARG, "top = %d outside [0, %d]", top, ALOCO_MAX_TOP);
    if (!grad) return fail(ALOCO_ERR_ARG, "NULL grad");
    bool over;
    if ((rc = take_grad(tokens, grad, &a, &s, &over)) != ALOCO_OK) return rc;
    if (a.n == 0) return done();
    const size_t each = (size_t)a.n * 4;
    if (top == 0) d_top = nullptr;
    s.add("stats", stats, 2 * each, 8, false);
    if (d_logp) s.add("d_logp", d_logp, each, 4, false);
    if (d_entropy) {
        s.add("d_entropy", d_entropy, each, 4, false);
        s.add("entropy", entropy, each, 4, false);
    }
    if (d_top) {
        s.add("d_top", d_top, each * top, 4, false);
        s.add("top_ids", top_ids, each * top, 4, false);
    }
    int sms;
    if ((rc = check_buffers(s, over, &sms)) != ALOCO_OK) return rc;
    aloco::ScoresArgs b;
    take_scores(tokens, a, top, &b);
    b.stats_in = reinterpret_cast<const float2 *>(stats);
    b.entropy_in = entropy;
    b.d_logp = d_logp;
    b.d_entropy = d_entropy;
    b.ids_in = top_ids;
    b.d_top = d_top;
    const cudaError_t e = aloco::launch_token_scores_grad(b, sms, stream_of(opts));
    return e == cudaSuccess ? done() : cuda_fail(e, "token scores' gradient");
}

int aloco_policy_loss(const aloco_tokens_t *tokens, const float *advantages,
                      const float *old_logp, const float *ref_logp, const float *weights,
                      const aloco_policy_cfg_t *cfg, float *terms, float *logp,
                      const aloco_logits_grad_t *grad, void *scratch, size_t scratch_bytes,
                      const aloco_opts_t *opts) {
    aloco::LogitsArgs a;
    Buffers s;
    int rc = take_tokens(tokens, &a, &s);
    if (rc != ALOCO_OK) return rc;
    if (!cfg) return fail(ALOCO_ERR_ARG, "NULL cfg");
    if (!(std::isfinite(cfg->clip_low) && cfg->clip_low >= 0.0) ||
        !(std::isfinite(cfg->clip_high) && cfg->clip_high >= 0.0))
        return fail(ALOCO_ERR_ARG, "clip_low = %g and clip_high = %g must be finite and >= 0",
                    cfg->clip_low, cfg->clip_high);
    if (!(std::isfinite(cfg->kl_coef) && cfg->kl_coef >= 0.0))
        return fail(ALOCO_ERR_ARG, "kl_coef = %g must be finite and >= 0", cfg->kl_coef);
    if (a.n > 0 && !ref_logp && cfg->kl_coef != 0.0)
        return fail(ALOCO_ERR_ARG, "kl_coef = %g needs ref_logp", cfg->kl_coef);
    const size_t each = (size_t)a.n * 4;
    s.add("advantages", advantages, each, 4, false);
    s.add("old_logp", old_logp, each, 4, false);
    if (ref_logp) s.add("ref_logp", ref_logp, each, 4, false);
    s.add("weights", weights, each, 4, false);
    s.add("terms", terms, 4 * sizeof(float), 4, true);
    s.add("logp", logp, each, 4, true);
    bool over;
    if ((rc = take_grad(tokens, grad, &a, &s, &over)) != ALOCO_OK) return rc;
    if ((rc = take_scratch(scratch, scratch_bytes, &a, &s)) != ALOCO_OK) return rc;
    a.adv = advantages;
    a.old = old_logp;
    a.ref = ref_logp;
    a.w = weights;
    a.lo = (float)(1.0 - cfg->clip_low);
    a.hi = (float)(1.0 + cfg->clip_high);
    a.kl = (float)cfg->kl_coef;
    a.logp = logp;
    a.terms_out = terms;
    int sms;
    if ((rc = check_buffers(s, over, &sms)) != ALOCO_OK) return rc;
    take_stall(&a);
    const cudaError_t e =
        (tokens->dtype == ALOCO_BF16 ? aloco::policy_loss_bf16 : aloco::policy_loss_f32)(a, sms, stream_of(opts));
    return e == cudaSuccess ? done() : cuda_fail(e, "policy loss");
}

int aloco_preference_loss(const aloco_tokens_t *tokens, const float *ref_logp,
                          const void *cu_seqlens, int32_t cu_bytes, int64_t pairs,
                          const aloco_preference_cfg_t *cfg, float *loss, float *log_ratios,
                          float *logp, const aloco_logits_grad_t *grad, void *scratch,
                          size_t scratch_bytes, const aloco_opts_t *opts) {
    aloco::LogitsArgs a;
    Buffers s;
    int rc = take_tokens(tokens, &a, &s);
    if (rc != ALOCO_OK) return rc;
    if (!cfg) return fail(ALOCO_ERR_ARG, "NULL cfg");
    if (!(std::isfinite(cfg->beta) && cfg->beta > 0.0))
        return fail(ALOCO_ERR_ARG, "beta = %g must be finite and > 0", cfg->beta);
    if (!(cfg->label_smoothing >= 0.0 && cfg->label_smoothing < 1.0))
        return fail(ALOCO_ERR_ARG, "label_smoothing = %g outside [0, 1)", cfg->label_smoothing);
    if (cu_bytes != 4 && cu_bytes != 8)
        return fail(ALOCO_ERR_ARG, "cu_bytes = %d must be 4 or 8", cu_bytes);
    if (pairs < 0 || pairs > std::numeric_limits<int32_t>::max() / 4)
        return fail(ALOCO_ERR_ARG, "pairs = %lld out of range", (long long)pairs);
    const size_t each = (size_t)a.n * 4;
    if (ref_logp) s.add("ref_logp", ref_logp, each, 4, false);
    if (pairs)
        s.add("cu_seqlens", cu_seqlens, (size_t)(2 * pairs + 1) * cu_bytes, (size_t)cu_bytes,
              false);
    s.add("loss", loss, 4, 4, true);
    s.add("log_ratios", log_ratios, (size_t)pairs * 8, 4, true);
    s.add("logp", logp, each, 4, true);
    bool over;
    if ((rc = take_grad(tokens, grad, &a, &s, &over)) != ALOCO_OK) return rc;
    if ((rc = take_scratch(scratch, scratch_bytes, &a, &s)) != ALOCO_OK) return rc;
    a.ref = ref_logp;
    a.cu = cu_seqlens;
    a.cu_bytes = cu_bytes;
    a.pairs = pairs;
    a.beta = (float)cfg->beta;
    a.eps = (float)cfg->label_smoothing;
    a.per_pair = pairs ? (float)(cfg->beta / (double)pairs) : 0.f;
    a.loss = loss;
    a.ratios = log_ratios;
    a.logp = logp;
    int sms;
    if ((rc = check_buffers(s, over, &sms)) != ALOCO_OK) return rc;
    take_stall(&a);
    const cudaError_t e =
        (tokens->dtype == ALOCO_BF16 ? aloco::preference_loss_bf16 : aloco::preference_loss_f32)(a, sms, stream_of(opts));
    return e == cudaSuccess ? done() : cuda_fail(e, "preference loss");
}

}  // extern "C"

// ------------------------------------------------------------ gradient lists

struct aloco_grads {
    int device = -1;
    int sm_count = 0;
    int n_chunks = 0;
    char *dev = nullptr;           // chunk table, and scratch for callers with none
    size_t scratch_bytes = 0;      // ticket, factor and partial sums
    void *scratch = nullptr;
    aloco::GradArgs args;          // the table filled in
    int64_t total = 0;
    bool overlap = false;          // two tensors share memory
    std::vector<std::pair<uintptr_t, uintptr_t>> ranges;  // sorted [begin, end)
};

namespace {

int grads_create(const void *const *grads, const int64_t *sizes, const int32_t *dtypes,
                 int64_t n, aloco_grads_t **out) {
    *out = nullptr;
    int device, sms, rc;
    if ((rc = current_device(&device, &sms)) != ALOCO_OK) return rc;
    int64_t total = 0;
    std::vector<std::pair<uintptr_t, uintptr_t>> ranges;
    RangeCheck check;
    for (int64_t i = 0; i < n; ++i) {
        const size_t size = dtypes[i] == ALOCO_F32 ? 4 : 2;
        if (sizes[i] == 0) continue;
        if ((rc = check(grads[i], (size_t)sizes[i] * size, device, "grads",
                                      (int)std::min<int64_t>(i, INT32_MAX))) != ALOCO_OK)
            return rc;
        ranges.push_back({(uintptr_t)grads[i], (uintptr_t)grads[i] + (size_t)sizes[i] * size});
        total += sizes[i];
    }
    std::sort(ranges.begin(), ranges.end());
    bool overlap = false;
    for (size_t i = 1; i < ranges.size(); ++i)
        overlap = overlap || ranges[i].first < ranges[i - 1].second;

    // Stretches of equal length: some for every block of the norm pass, none
    // so short that its start and end outweigh it.
    int64_t len = total / (sms * 8) / 4096 * 4096;
    len = std::min<int64_t>(std::max<int64_t>(len, 4096), 32768);
    std::vector<aloco::GradChunk> chunks;
    int64_t at = 0;
    for (int64_t i = 0; i < n; ++i) {
        const size_t size = dtypes[i] == ALOCO_F32 ? 4 : 2;
        for (int64_t e = 0; e < sizes[i]; e += len)
            chunks.push_back({(char *)const_cast<void *>(grads[i]) + (size_t)e * size, at + e,
                              (int32_t)std::min(len, sizes[i] - e), dtypes[i] == ALOCO_BF16});
        at += sizes[i];
    }
    if (chunks.size() > (size_t)INT32_MAX / 2)
        return fail(ALOCO_ERR_ARG, "%zu stretches of gradients: too many", chunks.size());

    const size_t table = (chunks.size() * sizeof(aloco::GradChunk) + 255) / 256 * 256;
    const int blocks = aloco::grad_norm_blocks(sms, (int)chunks.size());
    const size_t scratch = (size_t)blocks * sizeof(aloco::GradPartial) + 16;
    const size_t bytes = table + scratch;
    char *dev = nullptr;
    cudaError_t e = cudaMalloc((void **)&dev, bytes);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(ALOCO_ERR_NOMEM, "gradient list cudaMalloc(%zu): %s", bytes,
                    cudaGetErrorString(e));
    }
    e = cudaMemset(dev, 0, bytes);
    if (e == cudaSuccess && !chunks.empty())
        e = cudaMemcpy(dev, chunks.data(), chunks.size() * sizeof(aloco::GradChunk),
                       cudaMemcpyHostToDevice);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    aloco_grads *h = e == cudaSuccess ? new (std::nothrow) aloco_grads : nullptr;
    if (!h) {
        cudaFree(dev);
        cudaGetLastError();
        return e == cudaSuccess ? fail(ALOCO_ERR_NOMEM, "gradient list: out of host memory")
                                : cuda_fail(e, "gradient list");
    }
    h->device = device;
    h->sm_count = sms;
    h->n_chunks = (int)chunks.size();
    h->dev = dev;
    h->total = total;
    h->overlap = overlap;
    h->ranges.swap(ranges);
    std::memset(&h->args, 0, sizeof h->args);
    h->args.chunks = reinterpret_cast<const aloco::GradChunk *>(dev);
    h->args.n_chunks = h->n_chunks;
    h->scratch_bytes = scratch;
    h->scratch = dev + table;
    *out = h;
    return done();
}

bool meet(const void *p, size_t m, const void *q, size_t n) {
    return (uintptr_t)p < (uintptr_t)q + n && (uintptr_t)q < (uintptr_t)p + m;
}

bool hits(const aloco_grads_t *g, const void *p, size_t bytes) {
    const uintptr_t a = (uintptr_t)p, b = a + bytes;
    for (const auto &r : g->ranges)
        if (a < r.second && r.first < b) return true;
    return false;
}

// What both operators check of the list, norm and scratch (null: the handle's
// own); fills in their arguments.
int take_list(const aloco_grads_t *g, float *norm, void *scratch, size_t scratch_bytes,
              RangeCheck *check, aloco::GradArgs *a) {
    if (!g) return fail(ALOCO_ERR_ARG, "NULL gradient list");
    if (!norm) return fail(ALOCO_ERR_ARG, "NULL norm");
    if ((uintptr_t)norm & 3) return fail(ALOCO_ERR_ARG, "norm: not aligned to 4 bytes");
    int device, sms, rc;
    if ((rc = current_device(&device, &sms)) != ALOCO_OK) return rc;
    if (device != g->device)
        return fail(ALOCO_ERR_ARG, "the gradient list lives on device %d, current device is %d",
                    g->device, device);
    if (hits(g, norm, 4)) return fail(ALOCO_ERR_ALIAS, "norm overlaps a gradient");
    if ((rc = (*check)(norm, 4, device, "norm")) != ALOCO_OK) return rc;
    if (scratch) {
        if (scratch_bytes < g->scratch_bytes)
            return fail(ALOCO_ERR_ARG, "scratch of %zu bytes, need %zu", scratch_bytes,
                        g->scratch_bytes);
        if ((uintptr_t)scratch & 15)
            return fail(ALOCO_ERR_ARG, "scratch: not aligned to 16 bytes");
        if (meet(norm, 4, scratch, g->scratch_bytes))
            return fail(ALOCO_ERR_ALIAS, "scratch and norm overlap");
        if (hits(g, scratch, g->scratch_bytes))
            return fail(ALOCO_ERR_ALIAS, "scratch overlaps a gradient");
        if ((rc = (*check)(scratch, g->scratch_bytes, device, "scratch")) != ALOCO_OK) return rc;
    } else {
        scratch = g->scratch;
    }
    *a = g->args;
    a->norm = norm;
    a->ticket = static_cast<unsigned int *>(scratch);
    a->factor = static_cast<float *>(scratch) + 1;
    a->partials = reinterpret_cast<aloco::GradPartial *>(static_cast<char *>(scratch) + 16);
    return ALOCO_OK;
}

// The norm's kernel.  The handle's own scratch, which calls that overlapped may
// have left with a count, begins anew in every call.
cudaError_t launch_norm(const aloco_grads_t *g, const aloco::GradArgs &a, bool own_scratch,
                        cudaStream_t stream) {
    if (own_scratch) {
        const cudaError_t e = cudaMemsetAsync(a.ticket, 0, sizeof *a.ticket, stream);
        if (e != cudaSuccess) return e;
    }
    return aloco::launch_grad_norm(a, g->sm_count, stream);
}

}  // namespace

extern "C" {

int aloco_grads_create(const void *const *grads, const int64_t *sizes, const int32_t *dtypes,
                       int64_t n, aloco_grads_t **out) {
    if (!out) return fail(ALOCO_ERR_ARG, "NULL out");
    if (n < 0) return fail(ALOCO_ERR_ARG, "n = %lld must be >= 0", (long long)n);
    if (n > 0 && (!grads || !sizes || !dtypes)) return fail(ALOCO_ERR_ARG, "NULL array");
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (dtypes[i] != ALOCO_F32 && dtypes[i] != ALOCO_BF16)
            return fail(ALOCO_ERR_ARG, "grads[%lld]: unknown dtype %d", (long long)i, dtypes[i]);
        if (sizes[i] < 0 || sizes[i] > std::numeric_limits<int64_t>::max() / 16 - total)
            return fail(ALOCO_ERR_ARG, "grads[%lld]: size %lld out of range", (long long)i,
                        (long long)sizes[i]);
        total += sizes[i];
        if (sizes[i] == 0) continue;
        if (!grads[i]) return fail(ALOCO_ERR_ARG, "NULL grads[%lld]", (long long)i);
        if ((uintptr_t)grads[i] & (dtypes[i] == ALOCO_F32 ? 3 : 1))
            return fail(ALOCO_ERR_ARG, "grads[%lld]: not aligned to its element", (long long)i);
    }
    try {
        return grads_create(grads, sizes, dtypes, n, out);
    } catch (const std::bad_alloc &) {
        return fail(ALOCO_ERR_NOMEM, "gradient list: out of host memory");
    }
}

void aloco_grads_destroy(aloco_grads_t *g) {
    if (!g) return;
    int prev = -1;
    cudaGetDevice(&prev);
    if (prev != g->device) cudaSetDevice(g->device);
    cudaDeviceSynchronize();
    cudaFree(g->dev);
    if (prev >= 0 && prev != g->device) cudaSetDevice(prev);
    cudaGetLastError();
    delete g;
}

size_t aloco_grads_scratch_bytes(const aloco_grads_t *g) { return g ? g->scratch_bytes : 0; }

int aloco_grad_norm_in(aloco_grads_t *g, float *norm, void *scratch, size_t scratch_bytes,
                       const aloco_opts_t *opts) {
    aloco::GradArgs a;
    RangeCheck check;
    const int rc = take_list(g, norm, scratch, scratch_bytes, &check, &a);
    if (rc != ALOCO_OK) return rc;
    const cudaError_t e = launch_norm(g, a, !scratch, stream_of(opts));
    return e == cudaSuccess ? done() : cuda_fail(e, "gradient norm");
}

int aloco_grad_norm(aloco_grads_t *g, float *norm, const aloco_opts_t *opts) {
    return aloco_grad_norm_in(g, norm, nullptr, 0, opts);
}

int aloco_clip_grads_in(aloco_grads_t *g, double max_norm, void *out, aloco_dtype out_dtype,
                        float *norm, void *scratch, size_t scratch_bytes,
                        const aloco_opts_t *opts) {
    aloco::GradArgs a;
    RangeCheck check;
    int rc = take_list(g, norm, scratch, scratch_bytes, &check, &a);
    if (rc != ALOCO_OK) return rc;
    if (!(std::isfinite((float)max_norm) && (float)max_norm > 0.f))
        return fail(ALOCO_ERR_ARG, "max_norm = %g must be finite and > 0 in fp32", max_norm);
    if (!out && g->overlap)
        return fail(ALOCO_ERR_ALIAS, "gradients overlap one another: they cannot be clipped "
                                     "in place");
    if (out && g->total > 0) {
        if (out_dtype != ALOCO_F32 && out_dtype != ALOCO_BF16)
            return fail(ALOCO_ERR_ARG, "unknown out_dtype %d", (int)out_dtype);
        const size_t size = out_dtype == ALOCO_F32 ? 4 : 2, bytes = (size_t)g->total * size;
        if ((uintptr_t)out & (size - 1))
            return fail(ALOCO_ERR_ARG, "out: not aligned to its element");
        if (meet(norm, 4, out, bytes)) return fail(ALOCO_ERR_ALIAS, "out and norm overlap");
        if (scratch && meet(scratch, g->scratch_bytes, out, bytes))
            return fail(ALOCO_ERR_ALIAS, "out and scratch overlap");
        if (hits(g, out, bytes)) return fail(ALOCO_ERR_ALIAS, "out overlaps a gradient");
        if ((rc = check(out, bytes, g->device, "out")) != ALOCO_OK) return rc;
    }
    a.max_norm = (float)max_norm;
    a.out = out;
    a.out_bf16 = out_dtype == ALOCO_BF16;
    cudaError_t e = launch_norm(g, a, !scratch, stream_of(opts));
    if (e == cudaSuccess) e = aloco::launch_grad_scale(a, g->sm_count, stream_of(opts));
    return e == cudaSuccess ? done() : cuda_fail(e, "gradient clipping");
}

int aloco_clip_grads(aloco_grads_t *g, double max_norm, void *out, aloco_dtype out_dtype,
                     float *norm, const aloco_opts_t *opts) {
    return aloco_clip_grads_in(g, max_norm, out, out_dtype, norm, nullptr, 0, opts);
}

}  // extern "C"
