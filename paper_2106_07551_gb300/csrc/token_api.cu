// C entry points of the token losses: argument checks, work space, launches.
#include <cmath>

#include "malib.h"
#include "token_common.cuh"

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

    int begin(const malib_token_batch* b, bool tokens) {
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
            if (tokens && !dev(b->tokens, 4)) return bad("tokens must be aligned device memory of the context's device");
        }
        if (!tokens && b->tokens) return bad("tokens must be NULL");
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
            const uintptr_t z0 = (uintptr_t)a.z, z1 = z0 + (uintptr_t)(((a.n - 1) * a.ld + a.V) * es);
            const uintptr_t g0 = (uintptr_t)g->grad, g1 = g0 + (uintptr_t)(((a.n - 1) * g->ld + a.V) * es);
            if (g0 < z1 && z0 < g1) return bad("gradient overlaps the logits other than in place");
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

    // Work space: counters, partial sums, and a row's statistics or share of them.
    int work() {
        static_assert(sizeof(TokenRow) == sizeof(RowSum), "one work space for either");
        void *fixed = nullptr, *rows = nullptr;
        const int r = ctx_token_work(ctx, a.n * (int64_t)sizeof(RowSum), &fixed, &rows);
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
    int r = c.begin(batch, true);
    if (r != MALIB_OK) return r;
    if (c.a.n == 0) return MALIB_OK;
    if (!c.opt(logp_out, 4) || !c.opt(entropy_out, 4))
        return c.bad("outputs must be device memory of the context's device");
    if ((r = c.work()) != MALIB_OK) return r;
    c.a.logp = logp_out;
    c.a.entropy = entropy_out;
    return c.done(launch_token_rows(c.a, kTokLogp, c.v.n_sm, c.v.stream), 1);
}

int malib_learn_token_ppo(malib_ctx* ctx, const malib_token_batch* batch, const malib_token_ppo* loss,
                          const malib_token_grad* grad, float* logp_out, float* stats_out) {
    Call c{ctx};
    if (!ctx_view(ctx, &c.v)) return MALIB_EINVAL;
    DevSel d(c.v.device);
    int r = c.begin(batch, true);
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
    if ((r = c.work()) != MALIB_OK) return r;
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
    int r = c.begin(batch, true);
    if (r != MALIB_OK) return r;
    if (!loss) return c.bad("loss is NULL");
    if (loss->n_pairs < 1 || loss->n_pairs > (1 << 30)) return c.bad("n_pairs must lie in [1, 2^30]");
    if (!(loss->beta > 0.0f) || std::isinf(loss->beta)) return c.bad("beta must be positive");
    if (!(loss->label_smoothing >= 0.0f && loss->label_smoothing < 1.0f)) return c.bad("label_smoothing must lie in [0, 1)");
    if ((r = c.gradient(grad)) != MALIB_OK) return r;
    if (!c.dev(loss->offsets, 8)) return c.bad("offsets must be aligned device memory of the context's device");
    if ((c.a.n > 0 && !c.opt(loss->ref_logp, 4)) || !c.opt(reward_out, 4) || !c.opt(stats_out, 4))
        return c.bad("ref_logp, reward_out and stats must be device memory of the context's device");
    if ((r = c.work()) != MALIB_OK) return r;
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
    int r = c.begin(batch, false);
    if (r != MALIB_OK) return r;
    if (!loss) return c.bad("loss is NULL");
    if (loss->top < 1 || loss->top > kTokenMaxTop) return c.bad("top must lie in [1, 1024]");
    if (!known(loss->teacher_dtype)) return c.bad("unknown teacher dtype");
    if ((r = c.gradient(grad)) != MALIB_OK || (r = c.weights(loss->weight)) != MALIB_OK) return r;
    if (c.a.n > 0 && (!c.dev(loss->ids, 4) || !c.dev(loss->teacher, elt_size(loss->teacher_dtype)) || !c.opt(loss_out, 4)))
        return c.bad("ids, teacher and loss_out must be aligned device memory of the context's device");
    if (!c.opt(stats_out, 4)) return c.bad("stats must be device memory of the context's device");
    if ((r = c.work()) != MALIB_OK) return r;
    c.a.ids = loss->ids;
    c.a.teacher = loss->teacher;
    c.a.tdtype = loss->teacher_dtype;
    c.a.top = loss->top;
    c.a.loss = loss_out;
    c.a.stats = stats_out;
    return c.done(launch_token_rows(c.a, kTokDistill, c.v.n_sm, c.v.stream), c.a.n > 0 || stats_out ? 1 : 0);
}

}  // extern "C"
