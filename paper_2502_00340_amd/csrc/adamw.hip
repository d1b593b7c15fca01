// AdamW over many tensors and the global norm of their gradients.  HBM-bound streams: per element the gradient and the states in,
// parameter and states out.
//
// The tensors' pointers travel in the kernel arguments (4 KB at most), so that a call needs no table in device memory and can be captured;
// a launch covers up to 40 tensors, a block CHUNK elements of one of them.  8-bit states have a scale for every 256 elements of a
// tensor, which a wave owns four at a time.
#include <initializer_list>

#include "common.h"

namespace cf {

constexpr int ADAM_TENSORS = 40, CHUNK = 4096, QBLOCK = 256;

struct AdamTensor {
    void* p;
    float* master;
    const void* g;
    void *m, *v;
    float *ms, *vs;
    int64_t n;
    float wd;
    int32_t end;            // blocks of this tensor and the ones before it
};
struct AdamArgs {
    double beta1, beta2, lr;
    float b1, b2, c1, c2;   // beta, 1 - beta
    float eps;
    int32_t step;
    uint32_t seed;
    int32_t first;          // number of the first tensor in the call
    float grad_scale, max_norm;
    const float *norm_dev, *lr_dev;
    const int32_t* step_dev;
    int32_t n_tensors;
    AdamTensor t[ADAM_TENSORS];
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

// A step's scalars, the same for all elements
struct AdamStep {
    float clip, size, inv_root, decay;      // of the gradient; lr / (1 - beta1^t); 1 / sqrt(1 - beta2^t); lr
    uint32_t step;
};

__device__ __forceinline__ double int_pow(double b, unsigned n) {
    double r = 1.;
    for (; n != 0; n >>= 1, b *= b)
        if (n & 1) r *= b;
    return r;
}

// false: the norm is not finite, the step is left out
__device__ __forceinline__ bool adam_step(const AdamArgs& a, AdamStep& s) {
    s.clip = a.grad_scale;
    if (a.norm_dev != nullptr) {
        const float norm = *a.norm_dev;
        if (!(norm - norm == 0.f)) return false;
        s.clip *= fminf(1.f, a.max_norm / (norm + 1e-6f));
    }
    const int t = a.step_dev != nullptr ? *a.step_dev : a.step;
    s.step = t < 1 ? 1 : t;
    const double lr = a.lr_dev != nullptr ? (double)*a.lr_dev : a.lr;
    s.decay = (float)lr;
    s.size = (float)(lr / (1. - int_pow(a.beta1, s.step)));
    s.inv_root = (float)(1. / sqrt(1. - int_pow(a.beta2, s.step)));
    return true;
}

// A product that is rounded by itself.  A moment is two rounded products and a rounded sum on purpose: which of the products a
// fused multiply-add would leave unrounded is the compiler's choice, and where a moment lies at a border of two 8-bit codes,
// the code, a whole step, would be too.
__device__ __forceinline__ float rounded(float a, float b) {
    float p = a * b;
    asm("" : "+v"(p));
    return p;
}

__device__ __forceinline__ void adam_one(const AdamArgs& a, const AdamStep& s, float wd, float g, float& w, float& m, float& v) {
    g = rounded(g, s.clip);
    m = rounded(a.b1, m) + rounded(a.c1, g);
    v = rounded(a.b2, v) + rounded(a.c2, rounded(g, g));
    w = w - s.decay * wd * w - s.size * m / (sqrtf(v) * s.inv_root + a.eps);
}

// four elements from i on, of which `left` exist
template <typename T> __device__ __forceinline__ void load4(const T* p, int64_t left, float (&o)[4]);
template <> __device__ __forceinline__ void load4<float>(const float* p, int64_t left, float (&o)[4]) {
    if (left >= 4) Vec<float>::load(p, o);
    else
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = e < left ? p[e] : 0.f;
}
template <> __device__ __forceinline__ void load4<bf16_t>(const bf16_t* p, int64_t left, float (&o)[4]) {
    if (left >= 4) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        o[0] = __uint_as_float(u.x << 16); o[1] = __uint_as_float(u.x & 0xFFFF0000u);
        o[2] = __uint_as_float(u.y << 16); o[3] = __uint_as_float(u.y & 0xFFFF0000u);
    } else
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = e < left ? bf16_to_f32(p[e]) : 0.f;
}
template <typename T> __device__ __forceinline__ void store4(T* p, int64_t left, const float (&o)[4]);
template <> __device__ __forceinline__ void store4<float>(float* p, int64_t left, const float (&o)[4]) {
    if (left >= 4) Vec<float>::store(p, o);
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = o[e];
}
template <> __device__ __forceinline__ void store4<bf16_t>(bf16_t* p, int64_t left, const float (&o)[4]) {
    if (left >= 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = (bf16_t)pack_bf16x2(o[e], 0.f);
}
// four e4m3 bytes
__device__ __forceinline__ unsigned load4_q(const unsigned char* p, int64_t left) {
    if (left >= 4) return *reinterpret_cast<const unsigned*>(p);
    unsigned r = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) r |= (unsigned)p[e] << (8 * e);
    return r;
}
__device__ __forceinline__ void store4_q(unsigned char* p, int64_t left, unsigned q) {
    if (left >= 4) { *reinterpret_cast<unsigned*>(p) = q; return; }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) p[e] = (unsigned char)(q >> (8 * e));
}
__device__ __forceinline__ void from_q(unsigned q, float scale, float (&o)[4]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
    o[0] = rounded(a[0], scale); o[1] = rounded(a[1], scale); o[2] = rounded(b[0], scale); o[3] = rounded(b[1], scale);
}
__device__ __forceinline__ unsigned to_q(const float (&x)[4]) {
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), true);
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
// 20 bits of a hash of an element (the finaliser of MurmurHash3 over its number and the tensor's key) as a number in [0, 1)
__device__ __forceinline__ float dither(uint32_t key, int64_t i) {
    uint32_t h = (uint32_t)i * 0x9E3779B1u + (uint32_t)(i >> 32) * 0x27D4EB2Fu + key;
    h = (h ^ (h >> 16)) * 0x85EBCA6Bu;
    h = (h ^ (h >> 13)) * 0xC2B2AE35u;
    return (float)((h ^ (h >> 16)) >> 12) * 0x1p-20f;
}
// r > 0 in units of the scale, rounded up to the next e4m3 value where what is cut off is 1 - u of a step or more; not to 0
__device__ __forceinline__ float round_up_by(float r, float u) {
    const unsigned e = __float_as_uint(fmaxf(r, 0x1p-6f)) & 0x7F800000u;
    const float ulp = __uint_as_float(e - (3u << 23)), inv = __uint_as_float((257u << 23) - e);     // 2^(e-3) and its inverse
    return r > 0.f ? fminf(fmaxf(floorf(r * inv + u) * ulp, 0x1p-9f), 448.f) : r;
}

template <typename P, typename G, bool MASTER, int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
    AdamStep s;
    if (!adam_step(a, s)) return;
    int k = 0;
    while ((int)blockIdx.x >= a.t[k].end) ++k;          // the grid has t[n_tensors - 1].end blocks
    const AdamTensor& t = a.t[k];
    const int64_t at = (int64_t)((int)blockIdx.x - (k > 0 ? a.t[k - 1].end : 0)) * CHUNK;
    const uint32_t key = a.seed + 0x85EBCA77u * (uint32_t)(a.first + k + 1) + 0xC2B2AE3Du * s.step;
#pragma unroll
    for (int r = 0; r < CHUNK / 1024; ++r) {
        const int64_t i = at + r * 1024 + threadIdx.x * 4, left = t.n - i;      // a wave has 256 elements: one scale
        float g[4], w[4], m[4], v[4];
        load4<G>((const G*)t.g + i, left, g);
        if (MASTER) load4<float>(t.master + i, left, w);
        else load4<P>((const P*)t.p + i, left, w);
        const int64_t blk = i / QBLOCK;
        if constexpr (BITS == 32) {
            load4<float>((const float*)t.m + i, left, m);
            load4<float>((const float*)t.v + i, left, v);
        } else {
            const bool any = blk * QBLOCK < t.n;
            from_q(load4_q((const unsigned char*)t.m + i, left), any ? t.ms[blk] : 0.f, m);
            from_q(load4_q((const unsigned char*)t.v + i, left), any ? t.vs[blk] : 0.f, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = rounded(v[e], v[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) adam_one(a, s, t.wd, g[e], w[e], m[e], v[e]);
        if (MASTER) store4<float>(t.master + i, left, w);
        store4<P>((P*)t.p + i, left, w);
        if constexpr (BITS == 32) {
            store4<float>((float*)t.m + i, left, m);
            store4<float>((float*)t.v + i, left, v);
        } else {
            float tm = 0.f, tv = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = sqrtf(v[e]);
                tm = fmaxf(tm, e < left ? fabsf(m[e]) : 0.f);
                tv = fmaxf(tv, e < left ? v[e] : 0.f);
            }
            tm = fmaxf(wave_max(tm), 0x1p-100f);
            tv = fmaxf(wave_max(tv), 0x1p-100f);
            const float im = rounded(1.f / tm, 448.f), iv = rounded(1.f / tv, 448.f);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[e] *= im;
                v[e] = round_up_by(rounded(v[e], iv), dither(key, i + e));
            }
            store4_q((unsigned char*)t.m + i, left, to_q(m));
            store4_q((unsigned char*)t.v + i, left, to_q(v));
            if ((threadIdx.x & 63) == 0 && left > 0) {
                t.ms[blk] = tm * (1.f / 448.f);
                t.vs[blk] = tv * (1.f / 448.f);
            }
        }
    }
}

// ---- global norm -----------------------------------------------------------
constexpr int NORM_TENSORS = 160, NORM_BLOCKS = 2048, NORM_CHUNK = 8192;
struct NormArgs {
    const void* g[NORM_TENSORS];
    int64_t n[NORM_TENSORS];
    int32_t end[NORM_TENSORS];      // chunks of this tensor and the ones before it
    int32_t n_tensors;
};
static_assert(sizeof(NormArgs) <= 4000, "kernel arguments");

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// partial[block]: sum of the squares of the block's chunks, in fp64, where no square overflows
template <typename G>
__global__ __launch_bounds__(256) void grad_norm_kernel(NormArgs a, double* __restrict__ partial) {
    __shared__ double red[4];
    double s = 0.;
    int k = 0;
    for (int c = blockIdx.x; c < a.end[a.n_tensors - 1]; c += gridDim.x) {
        while (c >= a.end[k]) ++k;
        const G* g = (const G*)a.g[k];
        const int64_t at = (int64_t)(c - (k > 0 ? a.end[k - 1] : 0)) * NORM_CHUNK;
#pragma unroll
        for (int r = 0; r < NORM_CHUNK / 1024; ++r) {
            const int64_t i = at + r * 1024 + threadIdx.x * 4;
            float x[4];
            load4<G>(g + i, a.n[k] - i, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) s += (double)x[e] * (double)x[e];
        }
    }
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) partial[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(256) void grad_norm_finish_kernel(const double* __restrict__ partial, int n, float scale, float* __restrict__ norm) {
    __shared__ double red[4];
    double s = 0.;
    for (int i = threadIdx.x; i < n; i += 256) s += partial[i];
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) *norm = (float)(sqrt(red[0] + red[1] + red[2] + red[3]) * fabs((double)scale));
}

}  // namespace cf

using namespace cf;

namespace {

bool off(const void* p, size_t a) { return (uintptr_t)p % a != 0; }
bool is_finite(double v) { return v - v == 0.; }

template <typename P, typename G, bool MASTER, int BITS>
void adamw_launch(const AdamArgs& a, hipStream_t st) {
    adamw_kernel<P, G, MASTER, BITS><<<a.t[a.n_tensors - 1].end, 256, 0, st>>>(a);
}
template <typename P, bool MASTER>
void adamw_dispatch(const AdamArgs& a, bool g32, bool bits8, hipStream_t st) {
    if (g32) bits8 ? adamw_launch<P, float, MASTER, 8>(a, st) : adamw_launch<P, float, MASTER, 32>(a, st);
    else bits8 ? adamw_launch<P, bf16_t, MASTER, 8>(a, st) : adamw_launch<P, bf16_t, MASTER, 32>(a, st);
}

}  // namespace

extern "C" {

cf_status cf_adamw_step(const cf_adamw_desc* d, const cf_adamw_tensor* tensors, int32_t n_tensors, cf_stream stream) {
    if (!d || (!tensors && n_tensors > 0)) return CF_ERR_NULL;
    for (int dt : {d->p_dtype, d->g_dtype})
        if (dt != CF_BF16 && dt != CF_F32) return CF_ERR_DTYPE;
    if (n_tensors < 0 || (d->state_bits != 8 && d->state_bits != 32)) return CF_ERR_SHAPE;
    if (!(d->lr >= 0.) || !is_finite(d->lr) || !(d->beta1 >= 0. && d->beta1 < 1.) || !(d->beta2 >= 0. && d->beta2 < 1.) || !((float)d->eps > 0.f) ||
        !is_finite(d->eps) || !is_finite(d->grad_scale) || (!d->step_dev && d->step < 1))
        return CF_ERR_SHAPE;
    if (d->norm_dev && !(d->max_norm > 0.f)) return CF_ERR_SHAPE;
    if (off(d->norm_dev, 4) || off(d->step_dev, 4) || off(d->lr_dev, 4)) return CF_ERR_SHAPE;
    const bool bits8 = d->state_bits == 8;
    bool master = false, plain = false;
    for (int k = 0; k < n_tensors; ++k) {
        const cf_adamw_tensor& t = tensors[k];
        if (t.n < 0 || t.n > (int64_t)1 << 35 || !is_finite(t.weight_decay) || t.weight_decay < 0.f) return CF_ERR_SHAPE;
        if (t.n == 0) continue;
        if (!t.p || !t.g || !t.m || !t.v || (bits8 && (!t.m_scale || !t.v_scale))) return CF_ERR_NULL;
        for (const void* p : {(const void*)t.p, (const void*)t.master, t.g, (const void*)t.m, (const void*)t.v})
            if (off(p, 16)) return CF_ERR_SHAPE;
        if (bits8 && (off(t.m_scale, 4) || off(t.v_scale, 4))) return CF_ERR_SHAPE;
        (t.master ? master : plain) = true;
    }
    // with or without master copies: one kind in a call
    if (master && (plain || d->p_dtype == CF_F32)) return CF_ERR_SHAPE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    AdamArgs a{};
    a.beta1 = d->beta1; a.beta2 = d->beta2; a.lr = d->lr;
    a.b1 = (float)d->beta1; a.b2 = (float)d->beta2; a.c1 = (float)(1. - d->beta1); a.c2 = (float)(1. - d->beta2);
    a.eps = (float)d->eps; a.step = d->step; a.seed = d->seed;
    a.grad_scale = d->grad_scale; a.max_norm = d->max_norm;
    a.norm_dev = d->norm_dev; a.lr_dev = d->lr_dev; a.step_dev = d->step_dev;
    int k = 0;
    while (k < n_tensors) {
        // as many tensors as the arguments hold; of 2^35 elements at most each, their blocks are counted in 32 bits
        a.first = k; a.n_tensors = 0;
        int64_t blocks = 0;
        for (; k < n_tensors && a.n_tensors < ADAM_TENSORS; ++k) {
            const cf_adamw_tensor& t = tensors[k];
            const int64_t b = (t.n + CHUNK - 1) / CHUNK;
            blocks += b;
            a.t[a.n_tensors++] = AdamTensor{t.p, t.master, t.g, t.m, t.v, t.m_scale, t.v_scale, t.n, t.weight_decay, (int32_t)blocks};
        }
        if (blocks == 0) continue;
        if (d->p_dtype == CF_F32) adamw_dispatch<float, false>(a, d->g_dtype == CF_F32, bits8, st);
        else if (master) adamw_dispatch<bf16_t, true>(a, d->g_dtype == CF_F32, bits8, st);
        else adamw_dispatch<bf16_t, false>(a, d->g_dtype == CF_F32, bits8, st);
        if (hipGetLastError() != hipSuccess) return CF_ERR_HIP;
    }
    return CF_OK;
}

size_t cf_grad_norm_workspace_bytes(int32_t n_tensors) {
    return n_tensors < 0 ? 0 : (size_t)(n_tensors > 0 ? ceil_div(n_tensors, NORM_TENSORS) : 1) * NORM_BLOCKS * sizeof(double);
}

cf_status cf_grad_norm(const void* const* grads, const int64_t* sizes, int32_t n_tensors, int32_t g_dtype, float grad_scale,
                       float* norm, void* ws, size_t ws_bytes, cf_stream stream) {
    if (!norm || (n_tensors > 0 && (!grads || !sizes))) return CF_ERR_NULL;
    if (g_dtype != CF_BF16 && g_dtype != CF_F32) return CF_ERR_DTYPE;
    if (n_tensors < 0 || !is_finite(grad_scale) || off(norm, 4)) return CF_ERR_SHAPE;
    for (int k = 0; k < n_tensors; ++k) {
        if (sizes[k] < 0 || sizes[k] > (int64_t)1 << 35) return CF_ERR_SHAPE;
        if (sizes[k] > 0 && !grads[k]) return CF_ERR_NULL;
        if (sizes[k] > 0 && off(grads[k], 16)) return CF_ERR_SHAPE;
    }
    if (!ws || off(ws, 16) || ws_bytes < cf_grad_norm_workspace_bytes(n_tensors)) return CF_ERR_WORKSPACE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    int partials = 0;
    for (int k0 = 0; k0 < n_tensors; k0 += NORM_TENSORS) {
        NormArgs a;
        a.n_tensors = n_tensors - k0 < NORM_TENSORS ? n_tensors - k0 : NORM_TENSORS;
        int64_t chunks = 0;
        for (int k = 0; k < a.n_tensors; ++k) {
            a.g[k] = grads[k0 + k];
            a.n[k] = sizes[k0 + k];
            chunks += (a.n[k] + NORM_CHUNK - 1) / NORM_CHUNK;
            a.end[k] = (int32_t)chunks;
        }
        if (chunks == 0) continue;
        const int grid = (int)(chunks < NORM_BLOCKS ? chunks : NORM_BLOCKS);
        double* out = (double*)ws + partials;
        if (g_dtype == CF_F32) grad_norm_kernel<float><<<grid, 256, 0, st>>>(a, out);
        else grad_norm_kernel<bf16_t><<<grid, 256, 0, st>>>(a, out);
        partials += grid;
    }
    grad_norm_finish_kernel<<<1, 256, 0, st>>>((const double*)ws, partials, grad_scale, norm);
    return hipGetLastError() == hipSuccess ? CF_OK : CF_ERR_HIP;
}

}  // extern "C"
