// Losses of kept tokens and their gradient towards the logits: one block per kept row reads the row twice, first for the running
// maximum and sum of the softmax, then (from the caches) for the gradient, which needs both.  HBM-bound: the kept rows of the
// logits in, the gradient out.
#include <math.h>

#include "common.h"

namespace cf {

constexpr float LOG2E = 1.4426950408889634f;

// 16 bytes at an address that need only be aligned to an element: rows of an odd vocabulary start anywhere
struct __attribute__((packed, aligned(2))) Bytes16 { unsigned x, y, z, w; };

template <typename T> __device__ __forceinline__ void widen(const Bytes16& b, float (&o)[Vec<T>::N]);
template <> __device__ __forceinline__ void widen<float>(const Bytes16& b, float (&o)[4]) {
    o[0] = __uint_as_float(b.x); o[1] = __uint_as_float(b.y); o[2] = __uint_as_float(b.z); o[3] = __uint_as_float(b.w);
}
template <> __device__ __forceinline__ void widen<bf16_t>(const Bytes16& b, float (&o)[8]) {
    const unsigned w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[2 * i] = __uint_as_float(w[i] << 16);
        o[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
template <typename T> __device__ __forceinline__ Bytes16 narrow(const float (&o)[Vec<T>::N]);
template <> __device__ __forceinline__ Bytes16 narrow<float>(const float (&o)[4]) {
    return Bytes16{__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3])};
}
template <> __device__ __forceinline__ Bytes16 narrow<bf16_t>(const float (&o)[8]) {
    return Bytes16{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]), pack_bf16x2(o[4], o[5]), pack_bf16x2(o[6], o[7])};
}
template <typename T> __device__ __forceinline__ T one_from_f32(float v);
template <> __device__ __forceinline__ float one_from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t one_from_f32<bf16_t>(float v) { return (bf16_t)pack_bf16x2(v, 0.f); }     // NaN stays NaN

struct LossArgs {
    const void* logits;
    int64_t stride;
    const int64_t* targets;
    const float *old_logp, *ref_logp, *adv, *weights;
    const int32_t *idx, *n_dev;
    int n_max, V;
    float scale;                // of the logits
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
__device__ __forceinline__ RowLoss row_loss(const LossArgs& a, float lp, int64_t row, float w, float inv_norm) {
    if (!a.policy) return RowLoss{make_float4(-w * lp, -w * lp, 0.f, 0.f), -w * inv_norm};
    const float A = a.adv[row], r = expf(lp - a.old_logp[row]);
    const float rc = fminf(fmaxf(r, a.lo), a.hi);
    const bool clipped = r * A > rc * A;
    const float first = clipped ? -rc * A : -r * A;
    float d = clipped ? 0.f : -r * A, k = 0.f;
    if (a.ref_logp != nullptr) {
        const float q = a.ref_logp[row] - lp, e = expm1f(q);        // exp(q) - 1 as such: k is the small rest of it
        k = e - q;
        d -= a.kl_coef * e;
    }
    return RowLoss{make_float4(w * (first + a.kl_coef * k), w * first, w * k, clipped ? w : 0.f), w * inv_norm * d};
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void token_loss_kernel(LossArgs a) {
    constexpr int VN = Vec<T>::N, WAVES = NT / 64;
    __shared__ float red[2 * WAVES];
    const int n_rows = live_rows(a.n_max, a.n_dev), j = blockIdx.x, tid = threadIdx.x;
    if (j >= n_rows) return;
    const int64_t row = a.idx != nullptr ? a.idx[j] : j;
    const T* l = (const T*)a.logits + row * a.stride;
    T* dl = a.dlogits != nullptr ? (T*)a.dlogits + (int64_t)j * a.dstride : nullptr;
    const int V = a.V, nv = V / VN;
    const int64_t y = a.targets[row];
    const float w = a.weights != nullptr ? a.weights[row] : 1.f;
    const float inv_norm = 1.f / (a.norm != 0.f ? a.norm : (float)n_rows);
    const float ks = a.scale * LOG2E;
    float lp = 0.f, m = 0.f, inv_s = 0.f;
    RowLoss rl{make_float4(0.f, 0.f, 0.f, 0.f), 0.f};
    const bool live = y >= 0 && y < V && w != 0.f;
    if (live) {
        const float ly = to_f32<T>(l[y]);
        float s = 0.f;
        m = -3.402823466e38f;
        auto take = [&](const float (&x)[VN]) {
            float t = m;
#pragma unroll
            for (int e = 0; e < VN; ++e) t = fmaxf(t, x[e]);
            s *= exp2f((m - t) * ks);
            m = t;
#pragma unroll
            for (int e = 0; e < VN; ++e) s += exp2f((x[e] - m) * ks);
        };
        for (int v = tid; v < nv; v += NT) {
            float x[VN];
            widen<T>(reinterpret_cast<const Bytes16*>(l)[v], x);
            take(x);
        }
        if (int c = nv * VN + tid; c < V) {
            float x[VN];
            x[0] = to_f32<T>(l[c]);
#pragma unroll
            for (int e = 1; e < VN; ++e) x[e] = -INFINITY;
            take(x);
        }
        float bm = m;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) bm = fmaxf(bm, __shfl_xor(bm, o, 64));
        s = wave_sum(s * exp2f((m - bm) * ks));
        if ((tid & 63) == 0) { red[tid >> 6] = bm; red[WAVES + (tid >> 6)] = s; }
        __syncthreads();
        m = red[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) m = fmaxf(m, red[i]);
        s = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) s += red[WAVES + i] * exp2f((red[i] - m) * ks);
        inv_s = 1.f / s;
        lp = (ly - m) * a.scale - logf(s);
        rl = row_loss(a, lp, row, w, inv_norm);
    }
    if (tid == 0) {
        if (a.logp != nullptr) a.logp[j] = lp;
        a.terms[j] = rl.terms;
    }
    if (dl == nullptr) return;
    if (!live || rl.coef == 0.f) {
        const Bytes16 zero{0u, 0u, 0u, 0u};
        for (int v = tid; v < nv; v += NT) reinterpret_cast<Bytes16*>(dl)[v] = zero;
        if (int c = nv * VN + tid; c < V) dl[c] = one_from_f32<T>(0.f);
        return;
    }
    const float cs = rl.coef * a.scale, neg = -cs * inv_s, at_y = -cs * expm1f(lp);
    for (int v = tid; v < nv; v += NT) {
        float x[VN];
        widen<T>(reinterpret_cast<const Bytes16*>(l)[v], x);
#pragma unroll
        for (int e = 0; e < VN; ++e) x[e] = neg * exp2f((x[e] - m) * ks);
        if (v == (int)y / VN) {
#pragma unroll
            for (int e = 0; e < VN; ++e) x[e] = e == (int)y % VN ? at_y : x[e];
        }
        reinterpret_cast<Bytes16*>(dl)[v] = narrow<T>(x);
    }
    if (int c = nv * VN + tid; c < V) dl[c] = one_from_f32<T>(c == (int)y ? at_y : neg * exp2f((to_f32<T>(l[c]) - m) * ks));
}

// stats = sums of the rows' terms over the live rows, in fp64 and in fixed order, over norm
__global__ __launch_bounds__(256) void loss_stats_kernel(const float4* __restrict__ terms, int n_max, const int32_t* __restrict__ n_dev,
                                                         float norm, float* __restrict__ stats) {
    __shared__ double red[4][4];
    const int n_rows = live_rows(n_max, n_dev);
    double s[4] = {0., 0., 0., 0.};
    for (int j = threadIdx.x; j < n_rows; j += 256) {
        const float4 t = terms[j];
        s[0] += t.x; s[1] += t.y; s[2] += t.z; s[3] += t.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s[i] += __shfl_xor(s[i], o, 64);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6][i] = s[i];
    }
    __syncthreads();
    if (threadIdx.x < 4) {
        const double t = red[0][threadIdx.x] + red[1][threadIdx.x] + red[2][threadIdx.x] + red[3][threadIdx.x];
        const double by = norm != 0.f ? (double)norm : (double)(n_rows > 0 ? n_rows : 1);
        stats[threadIdx.x] = (float)(t / by);
    }
}

}  // namespace cf

using namespace cf;

extern "C" {

size_t cf_token_loss_workspace_bytes(int32_t max_kept) {
    return max_kept < 0 ? 0 : align_up((size_t)(max_kept > 0 ? max_kept : 1) * sizeof(float4), 256);
}

cf_status cf_token_loss(const cf_loss_desc* desc, const void* logits, int64_t logits_stride, const int64_t* targets,
                        const float* old_logp, const float* ref_logp, const float* advantages, const float* weights,
                        const int32_t* idx, const int32_t* n_kept_dev, int32_t max_kept, void* dlogits, int64_t dlogits_stride,
                        float* logp, float* stats, void* ws, size_t ws_bytes, cf_stream stream) {
    if (!desc || !logits || !targets) return CF_ERR_NULL;
    if (!dlogits && !logp && !stats) return CF_ERR_NULL;
    if (desc->dtype != CF_BF16 && desc->dtype != CF_F32) return CF_ERR_DTYPE;
    const bool policy = desc->kind == CF_LOSS_POLICY;
    if (!policy && desc->kind != CF_LOSS_NLL) return CF_ERR_SHAPE;
    if (policy && (!old_logp || !advantages)) return CF_ERR_NULL;
    const float scale = desc->logit_scale == 0.f ? 1.f : desc->logit_scale;
    const auto finite = [](float v) { return v - v == 0.f; };
    if (desc->V <= 0 || max_kept < 0 || max_kept > (1 << 30)) return CF_ERR_SHAPE;
    if (!(scale > 0.f) || !finite(scale) || !finite(desc->norm)) return CF_ERR_SHAPE;
    if (policy && (!(desc->clip_lo >= 0.f && desc->clip_lo <= 1.f) || !(desc->clip_hi >= 0.f) || !finite(desc->kl_coef) ||
                   (!ref_logp && desc->kl_coef != 0.f)))
        return CF_ERR_SHAPE;
    const int64_t ls = logits_stride ? logits_stride : desc->V, ds = dlogits_stride ? dlogits_stride : desc->V;
    if (ls < desc->V || (dlogits && ds < desc->V)) return CF_ERR_SHAPE;
    const size_t e = dtype_size(desc->dtype);
    const auto off = [](const void* p, size_t a) { return p && (uintptr_t)p % a != 0; };
    if (off(logits, e) || off(dlogits, e) || off(targets, 8)) return CF_ERR_SHAPE;
    for (const void* p : {(const void*)old_logp, (const void*)ref_logp, (const void*)advantages, (const void*)weights, (const void*)idx,
                          (const void*)n_kept_dev, (const void*)logp, (const void*)stats})
        if (off(p, 4)) return CF_ERR_SHAPE;
    if (dlogits == logits && (idx || ls != ds)) return CF_ERR_SHAPE;     // a row would be written before another block has read it
    if (!ws || off(ws, 16) || ws_bytes < cf_token_loss_workspace_bytes(max_kept)) return CF_ERR_WORKSPACE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    LossArgs a{logits, ls, targets, old_logp, ref_logp, advantages, weights, idx, n_kept_dev, max_kept, desc->V, scale, policy,
               1.f - desc->clip_lo, 1.f + desc->clip_hi, policy ? desc->kl_coef : 0.f, desc->norm, dlogits, ds, logp, (float4*)ws};
    if (max_kept > 0) {
        if (desc->dtype == CF_F32) token_loss_kernel<float, 512><<<max_kept, 512, 0, st>>>(a);
        else token_loss_kernel<bf16_t, 512><<<max_kept, 512, 0, st>>>(a);
    }
    if (stats) loss_stats_kernel<<<1, 256, 0, st>>>((const float4*)ws, max_kept, n_kept_dev, desc->norm, stats);
    return hipGetLastError() == hipSuccess ? CF_OK : CF_ERR_HIP;
}

}  // extern "C"
