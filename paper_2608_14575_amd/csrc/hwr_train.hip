// Host side of what follows the products in a training step (hwr_ops.h): log probabilities and
// the logits' gradient.
#include <hip/hip_runtime.h>

#include "ops_context.hpp"
#include "ops_internal.hpp"

using namespace hwr;

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

}  // namespace

extern "C" {

hwr_status hwr_log_probs(hwr_ops *ops, const hwr_log_probs_args *a) {
    return c_boundary([&] { return log_probs(ops, a); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

hwr_status hwr_log_probs_grad(hwr_ops *ops, const hwr_log_probs_grad_args *a) {
    return c_boundary([&] { return log_probs_grad(ops, a); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

}  // extern "C"
