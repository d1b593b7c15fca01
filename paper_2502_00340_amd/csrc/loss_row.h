// What a kept row's log probability gives, shared by the losses from logits and from the head's input.
#pragma once

#include "common.h"

namespace cf {

struct LossArgs {
    const void* logits;
    int64_t stride;
    const int64_t* targets;
    const float *old_logp, *ref_logp, *adv, *weights;
    const int32_t *idx, *n_dev;
    int n_max, V;
    int first;              // row of the launch's first block
    float scale, k, klo;        // of the logits; times log2(e), and what rounding that left
    bool policy;
    float lo, hi, kl_coef;      // bounds of the ratio
    float norm;                 // 0: the number of live rows
    void* dlogits;
    int64_t dstride;
    float *logp;
    float4* terms;              // per live row, times its weight: loss, its first term, k, clipped or not
};

// What a row's log probability gives: the terms, and w/norm * dL/dlp
struct RowLoss {
    float4 terms;
    float coef;
};
struct RowHead {
    int row, y;             // y: -1 for a row that is left out
    const void* l;
    float w, ly, old, ref, adv;
    __device__ __forceinline__ bool live() const { return y >= 0; }
};
__device__ __forceinline__ RowLoss row_loss(const LossArgs& a, const RowHead& h, float lp, float inv_norm) {
    const float w = h.w;
    if (!a.policy) return RowLoss{make_float4(-w * lp, -w * lp, 0.f, 0.f), -w * inv_norm};
    // A ratio beyond fp32 counts for nothing without an advantage, and a divergence beyond it for nothing without a coefficient: neither makes 0 * inf
    const float A = h.adv, r = expf(lp - h.old), rA = A == 0.f && r == r ? 0.f : r * A;
    const float rc = fminf(fmaxf(r, a.lo), a.hi);
    const bool clipped = rA > rc * A;
    const float first = clipped ? -rc * A : -rA;
    float d = clipped ? 0.f : -rA, k = 0.f, kl = 0.f;
    if (a.ref_logp != nullptr) {
        const float q = h.ref - lp, e = expm1f(q);          // exp(q) - 1 as such: k is the small rest of it
        k = e < INFINITY ? e - q : e;
        if (a.kl_coef != 0.f) {
            kl = a.kl_coef * k;
            d -= a.kl_coef * e;
        }
    }
    return RowLoss{make_float4(w * (first + kl), w * first, w * k, clipped ? w : 0.f), w * inv_norm * d};
}

// The checks of a loss description and of what a policy loss needs
inline cf_status loss_desc_check(const cf_loss_desc* d, const float* old_logp, const float* ref_logp, const float* advantages, int32_t max_kept) {
    if (d->dtype != CF_BF16 && d->dtype != CF_F32) return CF_ERR_DTYPE;
    const bool policy = d->kind == CF_LOSS_POLICY;
    if (!policy && d->kind != CF_LOSS_NLL) return CF_ERR_SHAPE;
    if (policy && (!old_logp || !advantages)) return CF_ERR_NULL;
    const float scale = d->logit_scale == 0.f ? 1.f : d->logit_scale;
    const auto finite = [](float v) { return v - v == 0.f; };
    if (d->V <= 0 || d->V > (1 << 30) || max_kept < 0 || max_kept > (1 << 30)) return CF_ERR_SHAPE;
    if (!(scale > 0.f) || !finite((float)((double)scale * 1.4426950408889634)) || !finite(d->norm)) return CF_ERR_SHAPE;
    if (policy && (!(d->clip_lo >= 0.f && d->clip_lo <= 1.f) || !(d->clip_hi >= 0.f) || !finite(d->kl_coef) || (!ref_logp && d->kl_coef != 0.f)))
        return CF_ERR_SHAPE;
    return CF_OK;
}

// What the kernels take of a description that has passed them; logits, dlogits and terms are the caller's to fill in
inline LossArgs loss_args(const cf_loss_desc* d, const int64_t* targets, const float* old_logp, const float* ref_logp, const float* advantages,
                          const float* weights, const int32_t* idx, const int32_t* n_kept_dev, int32_t max_kept, float* logp) {
    LossArgs a{};
    const bool policy = d->kind == CF_LOSS_POLICY;
    a.scale = d->logit_scale == 0.f ? 1.f : d->logit_scale;
    const double k = (double)a.scale * 1.4426950408889634;
    a.k = (float)k;
    a.klo = (float)(k - (float)k);
    a.targets = targets; a.old_logp = old_logp; a.ref_logp = ref_logp; a.adv = advantages; a.weights = weights;
    a.idx = idx; a.n_dev = n_kept_dev; a.n_max = max_kept; a.V = d->V;
    a.policy = policy;
    a.lo = 1.f - d->clip_lo; a.hi = 1.f + d->clip_hi;
    a.kl_coef = policy ? d->kl_coef : 0.f;
    a.norm = d->norm;
    a.logp = logp;
    return a;
}

// stats = sums of the live rows' terms, in fp64 and in a fixed order, over norm (token_loss.hip)
void launch_loss_stats(const float4* terms, int n_max, const int32_t* n_dev, float norm, float* stats, hipStream_t st);

}  // namespace cf
