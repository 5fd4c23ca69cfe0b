// C entry points of the token losses: argument checks, work space, launches.
#include <cmath>

#include "malib.h"
#include "spans.h"
#include "token_common.cuh"
#include "token_rollout.h"

using namespace malib;

namespace {

constexpr int32_t kMaxVocab = 1 << 24;
constexpr int64_t kMaxRows = 1ll << 40;              // far past what memory holds; 16 bytes a row of work space

// Fixed work space: the counter, then the partial sums.
constexpr int64_t kPartOffset = 256;
static_assert(kPartOffset + (int64_t)kTokenMaxCtas * (int64_t)sizeof(Totals) <= kTokenFixedBytes, "token work space");

int elt_size(int32_t dtype) { return dtype == MALIB_F32 ? 4 : 2; }
bool known(int32_t dtype) { return dtype == MALIB_F32 || dtype == MALIB_BF16 || dtype == MALIB_F16; }

struct Call {
    malib_ctx* ctx;
    CtxView v{};
    TokenArgs a{};

    int bad(const char* what) { return ctx_fail(ctx, MALIB_EINVAL, what); }

    // Device memory of the context's device, aligned to its element.
    bool dev(const void* p, int align) const {
        return p && ((uintptr_t)p & (uintptr_t)(align - 1)) == 0 && ptr_where(p, v.device) == kPtrHere;
    }
    // The same, or NULL.
    bool opt(const void* p, int align) const { return !p || dev(p, align); }

    enum Tokens { kNoTokens, kNeedTokens, kMayTokens };

    int begin(const malib_token_batch* b, Tokens tokens) {
        a = TokenArgs{};
        if (!b) return bad("token batch is NULL");
        if (!known(b->dtype)) return bad("unknown logits dtype");
        if (b->vocab < 1 || b->vocab > kMaxVocab) return bad("vocab must lie in [1, 2^24]");
        if (b->n_rows < 0 || b->n_rows > kMaxRows) return bad("n_rows must lie in [0, 2^40]");
        if (b->ld != 0 && b->ld < b->vocab) return bad("logits row stride below vocab");
        const int64_t es = elt_size(b->dtype);
        if (b->n_rows > 0 && b->ld > INT64_MAX / es / b->n_rows) return bad("logits do not fit the address space");
        if (!(b->temperature >= 1e-6 && b->temperature <= 1e6)) return bad("temperature must lie in [1e-6, 1e6]");
        const double exact_k = 1.4426950408889634074 / b->temperature;
        const float k = (float)exact_k;
        if (b->n_rows > 0) {
            if (!dev(b->logits, (int)es)) return bad("logits must be aligned device memory of the context's device");
            if (tokens != kNoTokens && !(tokens == kMayTokens ? opt(b->tokens, 4) : dev(b->tokens, 4)))
                return bad("tokens must be aligned device memory of the context's device");
        }
        if (tokens == kNoTokens && b->tokens) return bad("tokens must be NULL");
        a.z = b->logits;
        a.ld = b->ld;
        a.n = b->n_rows;
        a.V = b->vocab;
        a.dtype = b->dtype;
        a.k = k;
        a.dk = (float)(0.69314718055994530942 * (exact_k / (double)k - 1.0));
        a.inv_t = (float)(1.0 / b->temperature);
        a.inv_t_lo = (float)(1.0 / b->temperature - (double)a.inv_t);
        a.tt = (float)(b->temperature * b->temperature);
        a.top_scale = (float)b->temperature;
        a.tokens = b->tokens;
        a.err = v.err;
        return MALIB_OK;
    }

    int gradient(const malib_token_grad* g) {
        a.gscale = 1.0f;
        if (!g || !g->grad) return MALIB_OK;
        const int64_t es = elt_size(a.dtype);
        if (std::isnan(g->scale) || std::isinf(g->scale)) return bad("gradient scale must be finite");
        a.gscale = g->scale;
        if (a.n == 0) return MALIB_OK;
        if (!dev(g->grad, (int)es)) return bad("gradient must be aligned device memory of the context's device");
        if (g->ld < a.V || g->ld > INT64_MAX / es / a.n) return bad("gradient row stride below vocab");
        if (g->grad != a.z || (g->ld != a.ld && a.n > 1)) {
            if (!apart(logits(), Span(g->grad, row_bytes(a.n, g->ld, a.V, es)))) return bad("gradient overlaps the logits other than in place");
        }
        a.g = g->grad;
        a.gld = g->ld;
        return MALIB_OK;
    }

    int weights(const float* w) {
        if (a.n > 0 && !opt(w, 4)) return bad("weight must be device memory of the context's device");
        a.weight = w;
        a.w0 = a.n > 0 ? (float)(1.0 / (double)a.n) : 0.0f;
        return MALIB_OK;
    }

    // The logits, and n values of 4 bytes.
    Span logits() const { return Span(a.z, row_bytes(a.n, a.ld, a.V, elt_size(a.dtype))); }
    Span four(const void* p, int64_t each = 1) const { return Span(p, (uint64_t)a.n * (uint64_t)each * 4); }

    // Work space: counters, partial sums, and the statistics, or shares of them, of n rows.
    int work(int64_t n) {
        static_assert(sizeof(TokenRow) == sizeof(RowSum), "one work space for either");
        void *fixed = nullptr, *rows = nullptr;
        const int r = ctx_token_work(ctx, n * (int64_t)sizeof(RowSum), &fixed, &rows);
        if (r != MALIB_OK) return r;
        a.ticket = static_cast<unsigned*>(fixed);
        a.claims = reinterpret_cast<unsigned long long*>(static_cast<uint8_t*>(fixed) + 128);
        a.part = reinterpret_cast<Totals*>(static_cast<uint8_t*>(fixed) + kPartOffset);
        a.row_sums = static_cast<RowSum*>(rows);
        return MALIB_OK;
    }

    // The launches' own status: the runtime's last error may be the caller's, and one of a launch
    // does not stay there for the caller's next check.
    int done(cudaError_t e, int launches) {
        if (e != cudaSuccess) {
            cudaGetLastError();
            return ctx_fail(ctx, MALIB_ECUDA, cudaGetErrorString(e));
        }
        ctx_count_launches(ctx, launches);
        return MALIB_OK;
    }
};

}  // namespace

extern "C" {

int malib_token_logprob(malib_ctx* ctx, const malib_token_batch* batch, float* logp_out, float* entropy_out) {
    Call c{ctx};
    if (!ctx_view(ctx, &c.v)) return MALIB_EINVAL;
    DevSel d(c.v.device);
    int r = c.begin(batch, Call::kNeedTokens);
    if (r != MALIB_OK) return r;
    if (c.a.n == 0) return MALIB_OK;
    if (!c.opt(logp_out, 4) || !c.opt(entropy_out, 4))
        return c.bad("outputs must be device memory of the context's device");
    if ((r = c.work(c.a.n)) != MALIB_OK) return r;
    c.a.logp = logp_out;
    c.a.entropy = entropy_out;
    return c.done(launch_token_rows(c.a, kTokLogp, c.v.n_sm, c.v.stream), 1);
}

int malib_learn_token_ppo(malib_ctx* ctx, const malib_token_batch* batch, const malib_token_ppo* loss,
                          const malib_token_grad* grad, float* logp_out, float* stats_out) {
    Call c{ctx};
    if (!ctx_view(ctx, &c.v)) return MALIB_EINVAL;
    DevSel d(c.v.device);
    int r = c.begin(batch, Call::kNeedTokens);
    if (r != MALIB_OK) return r;
    if (!loss) return c.bad("loss is NULL");
    if (!(loss->clip_low > 0.0f && loss->clip_low < 1.0f) || !(loss->clip_high > 0.0f) || std::isinf(loss->clip_high))
        return c.bad("clip_low must lie in (0, 1) and clip_high be positive");
    if (!(loss->kl_coef >= 0.0f) || !(loss->entropy_coef >= 0.0f) || std::isinf(loss->kl_coef) ||
        std::isinf(loss->entropy_coef))
        return c.bad("kl_coef and entropy_coef must be >= 0");
    if ((r = c.gradient(grad)) != MALIB_OK || (r = c.weights(loss->weight)) != MALIB_OK) return r;
    if (c.a.n > 0 && (!c.dev(loss->old_logp, 4) || !c.dev(loss->advantage, 4) || !c.opt(loss->ref_logp, 4) ||
                      !c.opt(logp_out, 4)))
        return c.bad("old_logp, advantage, ref_logp and logp_out must be device memory of the context's device");
    if (!c.opt(stats_out, 4)) return c.bad("stats must be device memory of the context's device");
    if ((r = c.work(c.a.n)) != MALIB_OK) return r;
    c.a.old_logp = loss->old_logp;
    c.a.adv = loss->advantage;
    c.a.ref = loss->ref_logp;
    c.a.ratio_lo = 1.0f - loss->clip_low;
    c.a.ratio_hi = 1.0f + loss->clip_high;
    c.a.kl = loss->kl_coef;
    c.a.ent = loss->entropy_coef;
    c.a.logp = logp_out;
    c.a.stats = stats_out;
    return c.done(launch_token_rows(c.a, kTokPpo, c.v.n_sm, c.v.stream), c.a.n > 0 || stats_out ? 1 : 0);
}

int malib_learn_token_pref(malib_ctx* ctx, const malib_token_batch* batch, const malib_token_pref* loss,
                           const malib_token_grad* grad, float* reward_out, float* stats_out) {
    Call c{ctx};
    if (!ctx_view(ctx, &c.v)) return MALIB_EINVAL;
    DevSel d(c.v.device);
    int r = c.begin(batch, Call::kNeedTokens);
    if (r != MALIB_OK) return r;
    if (!loss) return c.bad("loss is NULL");
    if (loss->n_pairs < 1 || loss->n_pairs > (1 << 30)) return c.bad("n_pairs must lie in [1, 2^30]");
    if (!(loss->beta > 0.0f) || std::isinf(loss->beta)) return c.bad("beta must be positive");
    if (!(loss->label_smoothing >= 0.0f && loss->label_smoothing < 1.0f)) return c.bad("label_smoothing must lie in [0, 1)");
    if ((r = c.gradient(grad)) != MALIB_OK) return r;
    if (!c.dev(loss->offsets, 8)) return c.bad("offsets must be aligned device memory of the context's device");
    if ((c.a.n > 0 && !c.opt(loss->ref_logp, 4)) || !c.opt(reward_out, 4) || !c.opt(stats_out, 4))
        return c.bad("ref_logp, reward_out and stats must be device memory of the context's device");
    if ((r = c.work(c.a.n)) != MALIB_OK) return r;
    c.a.rows = reinterpret_cast<TokenRow*>(c.a.row_sums);
    c.a.offsets = loss->offsets;
    c.a.n_pairs = loss->n_pairs;
    c.a.ref = loss->ref_logp;
    c.a.beta = loss->beta;
    c.a.smooth = loss->label_smoothing;
    c.a.reward = reward_out;
    c.a.stats = stats_out;
    return c.done(launch_token_pairs(c.a, c.v.n_sm, c.v.stream), 1 + (c.a.n > 0) + (c.a.n > 0 && c.a.g));
}

int malib_learn_token_distill(malib_ctx* ctx, const malib_token_batch* batch, const malib_token_distill* loss,
                              const malib_token_grad* grad, float* loss_out, float* stats_out) {
    Call c{ctx};
    if (!ctx_view(ctx, &c.v)) return MALIB_EINVAL;
    DevSel d(c.v.device);
    int r = c.begin(batch, Call::kNoTokens);
    if (r != MALIB_OK) return r;
    if (!loss) return c.bad("loss is NULL");
    if (loss->top < 1 || loss->top > kTokenMaxTop) return c.bad("top must lie in [1, 1024]");
    if (!known(loss->teacher_dtype)) return c.bad("unknown teacher dtype");
    if ((r = c.gradient(grad)) != MALIB_OK || (r = c.weights(loss->weight)) != MALIB_OK) return r;
    if (c.a.n > 0 && (!c.dev(loss->ids, 4) || !c.dev(loss->teacher, elt_size(loss->teacher_dtype)) || !c.opt(loss_out, 4)))
        return c.bad("ids, teacher and loss_out must be aligned device memory of the context's device");
    if (!c.opt(stats_out, 4)) return c.bad("stats must be device memory of the context's device");
    if ((r = c.work(c.a.n)) != MALIB_OK) return r;
    c.a.ids = loss->ids;
    c.a.teacher = loss->teacher;
    c.a.tdtype = loss->teacher_dtype;
    c.a.top = loss->top;
    c.a.loss = loss_out;
    c.a.stats = stats_out;
    return c.done(launch_token_rows(c.a, kTokDistill, c.v.n_sm, c.v.stream), c.a.n > 0 || stats_out ? 1 : 0);
}

int malib_token_top(malib_ctx* ctx, const malib_token_batch* batch, const malib_token_list* out) {
    Call c{ctx};
    if (!ctx_view(ctx, &c.v)) return MALIB_EINVAL;
    DevSel d(c.v.device);
    int r = c.begin(batch, Call::kMayTokens);
    if (r != MALIB_OK) return r;
    if (!out) return c.bad("list is NULL");
    if (out->top < 1 || out->top > kTokenMaxTop) return c.bad("top must lie in [1, 1024]");
    if ((out->logp || out->rank) && !batch->tokens) return c.bad("logp and rank need tokens");
    if (c.a.n == 0) return MALIB_OK;
    if (c.a.n > INT64_MAX / 4 / out->top) return c.bad("the lists do not fit the address space");
    if (!c.dev(out->ids, 4) || !c.dev(out->top_logp, 4) || !c.opt(out->logp, 4) || !c.opt(out->entropy, 4) ||
        !c.opt(out->rank, 4))
        return c.bad("outputs must be device memory of the context's device");
    const Span in[] = {c.logits(), c.four(batch->tokens)};
    const Span outs[] = {c.four(out->ids, out->top), c.four(out->top_logp, out->top), c.four(out->logp), c.four(out->entropy),
                         c.four(out->rank)};
    if (!all_apart(outs, in)) return c.bad("an output overlaps an input or another output");
    ListArgs a{c.a};
    a.K = out->top;
    a.top_ids = out->ids;
    a.top_logp = out->top_logp;
    a.logp = out->logp;
    a.entropy = out->entropy;
    a.rank = out->rank;
    return c.done(launch_token_list(a, kListTop, c.v.n_sm, c.v.stream), 1);
}

int malib_token_sample(malib_ctx* ctx, const malib_token_batch* batch, const malib_token_draw* draw, int32_t* token_out,
                       float* logp_out, float* entropy_out, float* draw_logp_out) {
    Call c{ctx};
    if (!ctx_view(ctx, &c.v)) return MALIB_EINVAL;
    DevSel d(c.v.device);
    int r = c.begin(batch, Call::kMayTokens);
    if (r != MALIB_OK) return r;
    if (!draw) return c.bad("draw is NULL");
    if (draw->top_k < 0 || draw->top_k > kTokenMaxTop) return c.bad("top_k must lie in [0, 1024]");
    if (!(draw->top_p > 0.0f && draw->top_p <= 1.0f)) return c.bad("top_p must lie in (0, 1]");
    if (draw->top_k == 0 && draw->top_p < 1.0f) return c.bad("top_p below 1 needs top_k");
    if (draw->agent >> 31) return c.bad("agent must lie below 2^31");
    if (c.a.n == 0) return MALIB_OK;
    if (draw->uniform ? !c.dev(draw->uniform, 4) : !c.dev(draw->sequence, 8) || !c.dev(draw->step, 4))
        return c.bad("uniform, or sequence and step, must be aligned device memory of the context's device");
    if (!c.opt(token_out, 4) || !c.opt(logp_out, 4) || !c.opt(entropy_out, 4) || !c.opt(draw_logp_out, 4))
        return c.bad("outputs must be device memory of the context's device");
    // (tokens may be drawn in place)
    const Span in[] = {c.logits(), c.four(batch->tokens == token_out ? nullptr : batch->tokens), c.four(draw->uniform),
                       c.four(draw->uniform ? nullptr : draw->sequence, 2), c.four(draw->uniform ? nullptr : draw->step)};
    const Span outs[] = {c.four(token_out), c.four(logp_out), c.four(entropy_out), c.four(draw_logp_out)};
    if (!all_apart(outs, in)) return c.bad("an output overlaps an input or another output");
    if ((r = c.work(0)) != MALIB_OK) return r;
    ListArgs a{c.a};
    a.K = draw->top_k;
    a.drawn = token_out;
    a.logp = logp_out;
    a.entropy = entropy_out;
    a.draw_logp = draw_logp_out;
    a.uniform = draw->uniform;
    a.sequence = draw->sequence;
    a.step = draw->step;
    a.seed = draw->seed;
    a.agent = draw->agent;
    a.top_p = draw->top_p;
    return c.done(launch_token_list(a, draw->top_k ? kListDraw : kListDrawAll, c.v.n_sm, c.v.stream), 1);
}

int malib_learn_token_scores(malib_ctx* ctx, const malib_token_batch* batch, const malib_token_scores* scores,
                             const malib_token_grad* grad) {
    Call c{ctx};
    if (!ctx_view(ctx, &c.v)) return MALIB_EINVAL;
    DevSel d(c.v.device);
    int r = c.begin(batch, Call::kNeedTokens);
    if (r != MALIB_OK) return r;
    if (!scores) return c.bad("scores is NULL");
    if (c.a.n > 0 && !scores->logp_grad && !scores->entropy_grad && !scores->ids) return c.bad("no slopes are given");
    if (scores->ids && (scores->top < 1 || scores->top > kTokenMaxTop)) return c.bad("top must lie in [1, 1024]");
    if (!scores->ids && scores->top_grad) return c.bad("top_grad needs ids");
    if (!grad || (c.a.n > 0 && !grad->grad)) return c.bad("gradient is NULL");
    if ((r = c.gradient(grad)) != MALIB_OK) return r;
    if (c.a.n == 0) return MALIB_OK;
    if (!c.opt(scores->logp_grad, 4) || !c.opt(scores->entropy_grad, 4) || !c.opt(scores->ids, 4) ||
        (scores->ids && !c.dev(scores->top_grad, 4)))
        return c.bad("slopes and ids must be aligned device memory of the context's device");
    const Span in[] = {c.four(batch->tokens), c.four(scores->logp_grad), c.four(scores->entropy_grad),
                       c.four(scores->ids, scores->top), c.four(scores->ids ? scores->top_grad : nullptr, scores->top)};
    const Span outs[] = {Span(c.a.g, row_bytes(c.a.n, c.a.gld, c.a.V, elt_size(c.a.dtype)))};
    if (!all_apart(outs, in)) return c.bad("gradient overlaps tokens, ids or slopes");
    if ((r = c.work(0)) != MALIB_OK) return r;
    c.a.logp_grad = scores->logp_grad;
    c.a.entropy_grad = scores->entropy_grad;
    c.a.ids = scores->ids;
    c.a.list_grad = scores->top_grad;
    c.a.top = scores->ids ? scores->top : 0;
    return c.done(launch_token_rows(c.a, scores->ids ? kTokScoresList : kTokScores, c.v.n_sm, c.v.stream), 1);
}

int malib_dropout(malib_ctx* ctx, const malib_dropout_batch* b) {
    Call c{ctx};
    if (!ctx_view(ctx, &c.v)) return MALIB_EINVAL;
    DevSel d(c.v.device);
    if (!b) return c.bad("dropout batch is NULL");
    if (!known(b->dtype)) return c.bad("unknown dtype");
    if (b->dim < 1 || b->dim > (1 << 19)) return c.bad("dim must lie in [1, 524288]");
    if (b->n_rows < 0 || b->n_rows > kMaxRows) return c.bad("n_rows must lie in [0, 2^40]");
    if (!(b->p >= 0.0 && b->p <= 65535.0 / 65536.0)) return c.bad("p must lie in [0, 1 - 2^-16]");
    if (b->site >> 15) return c.bad("site must lie below 2^15");
    const int64_t n = b->n_rows, es = elt_size(b->dtype), most = n > 0 ? INT64_MAX / es / n : INT64_MAX;
    if ((b->ld_x != 0 && b->ld_x < b->dim) || (b->residual && b->ld_residual != 0 && b->ld_residual < b->dim) ||
        b->ld_out < b->dim || b->ld_x > most || (b->residual && b->ld_residual > most) || b->ld_out > most)
        return c.bad("row stride below dim, or rows past the address space");
    if (n == 0) return MALIB_OK;
    if (!c.dev(b->x, (int)es) || !c.opt(b->residual, (int)es) || !c.dev(b->out, (int)es))
        return c.bad("x, residual and out must be aligned device memory of the context's device");
    if (!c.dev(b->sequence, 8) || !c.dev(b->step, 4))
        return c.bad("sequence and step must be aligned device memory of the context's device");
    const Span out(b->out, row_bytes(n, b->ld_out, b->dim, es));
    const auto beside = [&](const void* in, int64_t ld) {
        return !in || (in == b->out && (ld == b->ld_out || n == 1)) || apart(Span(in, row_bytes(n, ld, b->dim, es)), out);
    };
    if (!beside(b->x, b->ld_x) || !beside(b->residual, b->ld_residual)) return c.bad("out overlaps x or residual other than in place");
    if (!apart(out, Span(b->sequence, (uint64_t)n * 8)) || !apart(out, Span(b->step, (uint64_t)n * 4)))
        return c.bad("out overlaps sequence or step");
    DropArgs a{};
    a.x = b->x;
    a.residual = b->residual;
    a.out = b->out;
    a.n = n;
    a.ld_x = b->ld_x;
    a.ld_res = b->ld_residual;
    a.ld_out = b->ld_out;
    a.d = b->dim;
    a.dtype = b->dtype;
    a.sequence = b->sequence;
    a.step = b->step;
    a.seed = b->seed;
    a.counter = 1u << 31 | b->site << 16;
    a.least = (uint32_t)(b->p * 65536.0 + 0.5);
    a.scale = (float)(65536.0 / (65536.0 - (double)a.least));
    return c.done(launch_dropout(a, c.v.n_sm, c.v.stream), 1);
}

}  // extern "C"
