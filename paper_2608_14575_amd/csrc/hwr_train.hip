// Host side of what follows the products in a training step (hwr_ops.h): log probabilities,
// the logits' gradient, and the step of the weights.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <memory>

#include "ops_context.hpp"
#include "ops_internal.hpp"

using namespace hwr;

struct hwr_adamw {
    int dev = 0;
    bool bf16 = false, master = false, states8 = false;
    int n_tensors = 0, n_chunks = 0;
    char *memory = nullptr;       // coefficients, tensors, the chunks' tensors
    AdamwCoef *coef() const { return reinterpret_cast<AdamwCoef *>(memory); }
};

namespace {

constexpr int kMaxTokens = 1 << 24;          // width of a row of logits
constexpr float kLeastScale = 0x1p-64f, kMostScale = 0x1p64f;

const char *check_logits(int32_t dtype, int32_t n, int32_t m, float scale) {
    if (dtype != HWR_F32 && dtype != HWR_BF16) return "unknown dtype";
    if (n < 0) return "n < 0";
    if (m < 1 || m > kMaxTokens) return "m outside 1..16777216";
    if (!(scale >= kLeastScale && scale <= kMostScale)) return "scale outside 2^-64..2^64";
    return nullptr;
}

hwr_status log_probs(hwr_ops *c, const hwr_log_probs_args *a) {
    if (!c) return invalid(nullptr, "ops is NULL");
    if (!a) return invalid(c, "arguments are NULL");
    if (const char *m = check_logits(a->dtype, a->n, a->m, a->scale)) return invalid(c, m);
    if (a->top < 0 || a->top > kMaxTop || a->top > a->m) return invalid(c, "top outside 0..32, or above m");
    if (bad_ld(a->ldx, a->m)) return invalid(c, "a row stride is smaller than the row");
    const bool tops = a->top_logp || a->top_token;
    if (tops != (a->top > 0) && a->n > 0) return invalid(c, "top_logp or top_token are required with top > 0, and only then");
    if (a->n == 0) return HWR_OK;
    if (!a->x || (a->logp && !a->token)) return invalid(c, "x is required, and token for logp");
    if (!a->logp && !a->lse && !a->entropy && !tops) return invalid(c, "no output");
    if (misaligned(a->dtype, {a->x}) || misaligned(HWR_F32, {a->token, a->logp, a->lse, a->entropy, a->top_logp, a->top_token}))
        return invalid(c, "a pointer is not aligned to its elements");
    OPS_ON_DEVICE(c, c->dev);
    const bool bf16 = a->dtype == HWR_BF16;
    ProbsArgs p{};
    p.n = a->n;
    p.m = a->m;
    p.top = a->top;
    p.scale = a->scale;
    p.x = a->x;
    p.ldx = dense(a->ldx, a->m);
    p.token = a->token;
    p.logp = a->logp;
    p.lse = a->lse;
    p.entropy = a->entropy;
    p.top_logp = a->top_logp;
    p.top_token = a->top_token;
    p.parts = probs_parts(bf16, a->n, a->m, c->cus);
    char *ws = nullptr;
    if (hwr_status st = workspace(c, probs_bytes(p), &ws)) return st;
    p.partial = ws;
    p.arrived = c->arrived;
    OPS_HIP(c, launch_probs(bf16, p, c->stream));
    return HWR_OK;
}

hwr_status log_probs_grad(hwr_ops *c, const hwr_log_probs_grad_args *a) {
    if (!c) return invalid(nullptr, "ops is NULL");
    if (!a) return invalid(c, "arguments are NULL");
    if (const char *m = check_logits(a->dtype, a->n, a->m, a->scale)) return invalid(c, m);
    if (bad_ld(a->ldx, a->m) || bad_ld(a->lddx, a->m)) return invalid(c, "a row stride is smaller than the row");
    if (a->n == 0) return HWR_OK;
    if (!a->x || !a->lse || !a->dx) return invalid(c, "x, lse and dx are required");
    if (a->dlogp && !a->token) return invalid(c, "token is required with dlogp");
    if (!a->entropy != !a->dentropy) return invalid(c, "entropy and dentropy go together");
    if (!a->dlogp && !a->dentropy) return invalid(c, "dlogp or dentropy is required");
    if (misaligned(a->dtype, {a->x, a->dx}) || misaligned(HWR_F32, {a->token, a->lse, a->dlogp, a->entropy, a->dentropy}))
        return invalid(c, "a pointer is not aligned to its elements");
    if (a->dx == a->x && dense(a->ldx, a->m) != dense(a->lddx, a->m) && a->n > 1)
        return invalid(c, "dx in place of x has to have its row stride");
    OPS_ON_DEVICE(c, c->dev);
    ProbsGradArgs p{};
    p.n = a->n;
    p.m = a->m;
    p.scale = a->scale;
    p.x = a->x;
    p.ldx = dense(a->ldx, a->m);
    p.token = a->token;
    p.lse = a->lse;
    p.dlogp = a->dlogp;
    p.entropy = a->entropy;
    p.dentropy = a->dentropy;
    p.dx = a->dx;
    p.lddx = dense(a->lddx, a->m);
    OPS_HIP(c, launch_probs_grad(a->dtype == HWR_BF16, p, c->stream));
    return HWR_OK;
}

// ---------------------------------------------------------------- AdamW
constexpr uint64_t kCoefBytes = 256;
constexpr int kMaxTensors = 1 << 20;
constexpr int64_t kMaxValues = int64_t{1} << 40;

// Bytes that a step reads or writes: [at, end).
struct Range {
    uintptr_t at, end;
    bool written;
};

hwr_status adamw_init(hwr_ops *c, const hwr_adamw_config *f, hwr_adamw **out) {
    if (!c) return invalid(nullptr, "ops is NULL");
    if (!out) return invalid(c, "out is NULL");
    *out = nullptr;
    if (!f) return invalid(c, "config is NULL");
    if (f->dtype != HWR_F32 && f->dtype != HWR_BF16) return invalid(c, "unknown dtype");
    if (f->bits != 8 && f->bits != 32) return invalid(c, "bits other than 8 and 32");
    if (f->n_tensors < 0 || f->n_tensors > kMaxTensors) return invalid(c, "n_tensors outside 0..1048576");
    if (f->n_tensors > 0 && !f->tensors) return invalid(c, "tensors is NULL");
    const bool bf16 = f->dtype == HWR_BF16, states8 = f->bits == 8;
    const int64_t size = bf16 ? 2 : 4;
    std::vector<AdamwTensor> tensors;
    int64_t chunks = 0;
    std::vector<Range> ranges;
    bool master = false, first = true;
    int64_t place = 0;
    for (int i = 0; i < f->n_tensors; ++i) {
        const hwr_adamw_tensor &t = f->tensors[i];
        const std::string which = "tensor " + std::to_string(i) + ": ";
        auto refuse = [&](const char *m) { return fail(c, HWR_ERR_INVALID_ARG, which + m); };
        if (t.count < 0 || t.count > kMaxValues) return refuse("count outside 0..2^40");
        if (t.count == 0) continue;
        if (!t.p || !t.g || !t.m || !t.v) return refuse("p, g, m and v are required");
        if (states8 != (t.m_scale != nullptr) || states8 != (t.v_scale != nullptr))
            return refuse("m_scale and v_scale are required with states of 8 bits, and only then");
        if (t.master && !bf16) return refuse("a master is for bf16 weights");
        if (!first && master != (t.master != nullptr)) return refuse("a master for some tensors and not for others");
        first = false;
        master = t.master != nullptr;
        if (misaligned(f->dtype, {t.p, t.g}) || misaligned(HWR_F32, {t.master, t.m_scale, t.v_scale}) ||
            (!states8 && misaligned(HWR_F32, {t.m, t.v})))
            return refuse("a pointer is not aligned to its elements");
        const int64_t blocks = (t.count + kAdamwBlock - 1) / kAdamwBlock, state = states8 ? 1 : 4;
        auto range = [&](const void *p, int64_t bytes, bool written) {
            const auto at = reinterpret_cast<uintptr_t>(p);
            if (p) ranges.push_back({at, at + bytes, written});
        };
        range(t.p, t.count * size, true);
        range(t.g, t.count * size, false);
        range(t.master, t.count * 4, true);
        range(t.m, t.count * state, true);
        range(t.v, t.count * state, true);
        range(t.m_scale, blocks * 4, true);
        range(t.v_scale, blocks * 4, true);
        const int64_t first_chunk = chunks;
        chunks += (t.count + kAdamwChunk - 1) / kAdamwChunk;
        if (chunks > INT32_MAX / 2) return refuse("more than 2^41 values in all");
        tensors.push_back({t.p, t.g, t.master, t.m, t.v, t.m_scale, t.v_scale, t.count, place, first_chunk});
        place += blocks * kAdamwBlock;
    }
    // nothing that is written may be a part of anything else
    std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.at < b.at; });
    uintptr_t end = 0, written_end = 0;           // of the ranges so far
    for (const Range &r : ranges) {
        if (r.at < (r.written ? end : written_end)) return invalid(c, "tensors overlap (gradients alone may)");
        end = std::max(end, r.end);
        if (r.written) written_end = std::max(written_end, r.end);
    }
    OPS_ON_DEVICE(c, c->dev);
    bool captured = false;
    OPS_HIP(c, is_captured(c, &captured));
    if (captured) return fail(c, HWR_ERR_STATE, "the stream is being captured: make it before");
    auto a = std::make_unique<hwr_adamw>();
    a->dev = c->dev;
    a->bf16 = bf16;
    a->master = master;
    a->states8 = states8;
    a->n_tensors = static_cast<int>(tensors.size());
    a->n_chunks = static_cast<int>(chunks);
    // one copy: the tensors, then the tensor of every chunk
    const uint64_t tb = tensors.size() * sizeof(AdamwTensor);
    std::vector<char> table(tb + chunks * sizeof(int));
    if (tb) std::memcpy(table.data(), tensors.data(), tb);
    int *of_chunk = reinterpret_cast<int *>(table.data() + tb);
    for (size_t i = 0; i < tensors.size(); ++i)
        std::fill(of_chunk + tensors[i].first, of_chunk + (i + 1 < tensors.size() ? tensors[i + 1].first : chunks), static_cast<int>(i));
    OPS_HIP(c, hipMalloc(reinterpret_cast<void **>(&a->memory), kCoefBytes + table.size()));
    const hipError_t e = tb ? hipMemcpy(a->memory + kCoefBytes, table.data(), table.size(), hipMemcpyHostToDevice) : hipSuccess;
    if (e != hipSuccess) {
        (void)hipFree(a->memory);
        return hip_fail(c, e, "hipMemcpy");
    }
    *out = a.release();
    return HWR_OK;
}

hwr_status adamw_step(hwr_ops *c, const hwr_adamw *w, const hwr_adamw_args *a) {
    if (!c) return invalid(nullptr, "ops is NULL");
    if (!w) return invalid(c, "adamw is NULL");
    if (!a) return invalid(c, "arguments are NULL");
    if (w->dev != c->dev) return invalid(c, "adamw belongs to another device");
    if (!(a->beta1 >= 0 && a->beta1 < 1 && a->beta2 >= 0 && a->beta2 < 1)) return invalid(c, "a beta outside [0, 1)");
    if (!(a->eps >= 0 && a->eps < 1)) return invalid(c, "eps outside [0, 1)");
    if (!std::isfinite(a->weight_decay) || a->weight_decay < 0) return invalid(c, "weight_decay is negative or not finite");
    if (!a->lr_device && (!std::isfinite(a->lr) || a->lr < 0)) return invalid(c, "lr is negative or not finite");
    if (!a->steps && a->step < 1) return invalid(c, "step < 1");
    if (a->lr_device && !a->steps) return invalid(c, "lr_device is for steps that are counted on the device");
    if (misaligned(HWR_F32, {a->lr_device}) || reinterpret_cast<uintptr_t>(a->steps) % 8)
        return invalid(c, "a pointer is not aligned to its elements");
    OPS_ON_DEVICE(c, c->dev);
    if (!a->steps) {
        bool captured = false;
        OPS_HIP(c, is_captured(c, &captured));
        if (captured)
            return fail(c, HWR_ERR_STATE, "a graph would repeat the same step: have the steps counted on the device");
    }
    AdamwArgs k{};
    k.tensors = reinterpret_cast<const AdamwTensor *>(w->memory + kCoefBytes);
    k.chunks = reinterpret_cast<const int *>(k.tensors + w->n_tensors);
    k.n_chunks = w->n_chunks;
    if (a->steps) {
        const AdamwRates r{a->lr, a->beta1, a->beta2, a->eps, a->weight_decay, a->seed, a->steps, a->lr_device};
        OPS_HIP(c, launch_adamw_coef(r, w->coef(), c->stream));
        k.coef_device = w->coef();
    } else {
        k.coef = adamw_coef(a->lr, a->beta1, a->beta2, a->eps, a->weight_decay, a->seed, a->step);
    }
    if (w->n_chunks == 0) return HWR_OK;
    OPS_HIP(c, launch_adamw(w->bf16, w->master, w->states8, k, c->stream));
    return HWR_OK;
}

}  // namespace

extern "C" {

hwr_status hwr_adamw_init(hwr_ops *ops, const hwr_adamw_config *config, hwr_adamw **out) {
    return c_boundary([&] { return adamw_init(ops, config, out); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

hwr_status hwr_adamw_step(hwr_ops *ops, hwr_adamw *adamw, const hwr_adamw_args *a) {
    return c_boundary([&] { return adamw_step(ops, adamw, a); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

void hwr_adamw_free(hwr_adamw *adamw) {
    if (!adamw) return;
    c_boundary(
        [&] {
            const OnDevice on_device(adamw->dev);
            (void)hipFree(adamw->memory);        // (waits for the device)
            delete adamw;
            return HWR_OK;
        },
        [](const char *) {});
}

hwr_status hwr_log_probs(hwr_ops *ops, const hwr_log_probs_args *a) {
    return c_boundary([&] { return log_probs(ops, a); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

hwr_status hwr_log_probs_grad(hwr_ops *ops, const hwr_log_probs_grad_args *a) {
    return c_boundary([&] { return log_probs_grad(ops, a); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

}  // extern "C"
