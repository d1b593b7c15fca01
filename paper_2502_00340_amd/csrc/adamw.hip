// AdamW over many tensors and the global norm of their gradients.  HBM-bound streams: per element the gradient and the states in,
// parameter and states out.
//
// The tensors' pointers travel in the kernel arguments (4 KB at most), so that a call needs no table in device memory and can be captured;
// a launch covers up to 40 tensors, a block CHUNK elements of one of them, a lane 8 of these.  8-bit states have a scale for every 256
// elements of a tensor, the ones of half a wave.
#include <initializer_list>
#include <type_traits>

#include "common.h"

namespace cf {

constexpr int ADAM_TENSORS = 40, LANE = 8, CHUNK = 256 * LANE, QBLOCK = 256;

struct AdamTensor {
    void* p;
    float* master;
    const void* g;
    void *m, *v;
    float *ms, *vs;
    int64_t n;
    float wd;
};
struct AdamArgs {
    int32_t end[ADAM_TENSORS];      // blocks of a tensor and the ones before it; of those behind the last INT_MAX
    AdamTensor t[ADAM_TENSORS];
    double beta1, beta2;
    float b1, b2, c1, c2;           // beta, 1 - beta
    float eps, lr, size, inv_root;  // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    uint32_t step, seed;
    int32_t first;                  // number of the first tensor in the call
    float grad_scale, max_norm;
    const float *norm_dev, *lr_dev;
    const int32_t* step_dev;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

// A step's scalars, the same for all elements
struct AdamStep {
    float clip, size, inv_root, lr;
    uint32_t step;
};

__host__ __device__ inline double int_pow(double b, unsigned n) {
    double r = 1.;
    for (; n != 0; n >>= 1, b *= b)
        if (n & 1) r *= b;
    return r;
}
__host__ __device__ inline void adam_scalars(double beta1, double beta2, double lr, unsigned step, float& size, float& inv_root) {
    size = (float)(lr / (1. - int_pow(beta1, step)));
    inv_root = (float)(1. / sqrt(1. - int_pow(beta2, step)));
}

// false: the norm is not finite, the step is left out
__device__ __forceinline__ bool adam_step(const AdamArgs& a, AdamStep& s) {
    s = AdamStep{a.grad_scale, a.size, a.inv_root, a.lr, a.step};
    if (a.norm_dev != nullptr) {
        const float norm = *a.norm_dev;
        if (!(norm - norm == 0.f)) return false;
        s.clip *= fminf(1.f, a.max_norm / (norm + 1e-6f));
    }
    if (a.step_dev != nullptr || a.lr_dev != nullptr) {
        if (a.lr_dev != nullptr) s.lr = *a.lr_dev;
        if (a.step_dev != nullptr) { const int t = *a.step_dev; s.step = t < 1 ? 1 : t; }
        adam_scalars(a.beta1, a.beta2, s.lr, s.step, s.size, s.inv_root);
    }
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

// Whether any lane of the wave has it: a branch of the whole wave, out of the way (900 -> 889 us for 218 M elements, where a branch of single lanes costs 8)
__device__ __forceinline__ bool seldom(bool c) { return __builtin_expect(__any(c), 0); }

// The square root to half a step: the hardware's, which is off by one and takes what is below the normal numbers for 0, and what a fused residual says is missing; a
// third of the instructions of sqrtf.  Below the normal numbers it comes out between 2^-64 and 2^-63, not below the root itself: what such a v has lost to fp32 does not
// divide a step.
__device__ __forceinline__ float root(float v) {
    const float s = fmaxf(__builtin_amdgcn_sqrtf(v), 0x1p-63f), r = fmaf(fmaf(-s, s, v), 0.5f * __builtin_amdgcn_rcpf(s), s);
    return s < INFINITY ? r : s;            // a square beyond fp32 makes an update of 0
}
// The root that an 8-bit state keeps: 0 of 0.  TINY: of any number, scaled up where it is small, else of normal ones.
template <bool TINY> __device__ __forceinline__ float kept_root(float v) {
    const int up = TINY && v < 0x1p-96f ? 32 : 0;
    const float x = TINY ? ldexpf(v, 2 * up) : v, s = __builtin_amdgcn_sqrtf(x);
    const float r = fmaf(fmaf(-s, s, x), 0.5f * __builtin_amdgcn_rcpf(fmaxf(s, 0x1p-70f)), s);
    return s < INFINITY ? TINY ? ldexpf(r, -up) : r : s;
}

// LANE elements from i on, of which `left` exist: all of them, unless TAIL
template <typename T, bool TAIL> __device__ __forceinline__ void load_lane(const T* p, int64_t left, float (&o)[LANE]) {
    if (TAIL && left < LANE) {
#pragma unroll
        for (int e = 0; e < LANE; ++e) o[e] = e < left ? to_f32<T>(p[e]) : 0.f;
        return;
    }
    constexpr int VN = Vec<T>::N;
#pragma unroll
    for (int q = 0; q < LANE / VN; ++q) Vec<T>::load(p + q * VN, reinterpret_cast<float (&)[VN]>(o[q * VN]));
}
// Past the caches, as all that a step writes.  For bf16 parameters 739 -> 733 us (8 bits, 218 M elements), and 192 -> 187 for the norm that comes next.
typedef unsigned u32x4a __attribute__((ext_vector_type(4)));
typedef unsigned u32x2a __attribute__((ext_vector_type(2)));
template <typename T, bool TAIL> __device__ __forceinline__ void store_lane(T* p, int64_t left, const float (&o)[LANE]) {
    constexpr int VN = Vec<T>::N;
    if (TAIL && left < LANE) {
#pragma unroll
        for (int e = 0; e < LANE; ++e)
            if (e < left) {
                if constexpr (VN == 8) p[e] = (T)pack_bf16x2(o[e], 0.f);
                else p[e] = o[e];
            }
        return;
    }
#pragma unroll
    for (int q = 0; q < LANE / VN; ++q) {
        u32x4a b;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if constexpr (VN == 8) b[e] = pack_bf16x2(o[2 * e], o[2 * e + 1]);
            else b[e] = __float_as_uint(o[4 * q + e]);
        __builtin_nontemporal_store(b, reinterpret_cast<u32x4a*>(p) + q);
    }
}
// LANE e4m3 bytes
template <bool TAIL> __device__ __forceinline__ uint2 load_bytes(const unsigned char* p, int64_t left) {
    if (!TAIL || left >= LANE) return *reinterpret_cast<const uint2*>(p);
    unsigned w[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < LANE; ++e)
        if (e < left) w[e / 4] |= (unsigned)p[e] << (8 * (e % 4));
    return make_uint2(w[0], w[1]);
}
template <bool TAIL> __device__ __forceinline__ void store_bytes(unsigned char* p, int64_t left, uint2 q) {
    if (!TAIL || left >= LANE) { __builtin_nontemporal_store(u32x2a{q.x, q.y}, reinterpret_cast<u32x2a*>(p)); return; }
#pragma unroll
    for (int e = 0; e < LANE; ++e)
        if (e < left) p[e] = (unsigned char)((e < 4 ? q.x : q.y) >> (8 * (e % 4)));
}
__device__ __forceinline__ void from_q(uint2 q, float scale, float (&o)[LANE]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const unsigned w[2] = {q.x, q.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        o[4 * i] = rounded(a[0], scale); o[4 * i + 1] = rounded(a[1], scale);
        o[4 * i + 2] = rounded(b[0], scale); o[4 * i + 3] = rounded(b[1], scale);
    }
}
// The same once more, from the bytes: what was converted before need not be held until then
__device__ __forceinline__ void again_from_q(uint2 q, float scale, float (&o)[LANE]) {
    asm("" : "+v"(q.x), "+v"(q.y));
    from_q(q, scale, o);
}
__device__ __forceinline__ uint2 to_q(const float (&x)[LANE]) {
    return make_uint2(__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), true),
                      __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false), true));
}
// over the 32 lanes of a scale
constexpr float TOP_MIN = 0x1p-100f;
__device__ __forceinline__ float block_max(float v) {
#pragma unroll
    for (int o = QBLOCK / LANE / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return fmaxf(v, TOP_MIN);
}
// A hash of an element: the published finishing steps of MurmurHash3 (two multiplications with shifts around them) over its number and the tensor's key.  Its
// upper 20 bits round v, the lower 12 m.
__device__ __forceinline__ uint32_t dither(uint32_t h) {
    h = (h ^ (h >> 16)) * 0x85EBCA6Bu;
    h = (h ^ (h >> 13)) * 0xC2B2AE35u;
    return h ^ (h >> 16);
}
// The distance of the e4m3 values from r (not negative, in units of the scale) on, and its inverse
__device__ __forceinline__ void e4m3_step(float r, float& ulp, float& inv) {
    const unsigned e = __float_as_uint(fmaxf(r, 0x1p-6f)) & 0x7F800000u;
    ulp = __uint_as_float(e - (3u << 23)), inv = __uint_as_float((257u << 23) - e);     // 2^(e-3)
}
// r in units of the scale, rounded up to the next e4m3 value where what is cut off and the dither make a step together; not to 0
__device__ __forceinline__ float round_up_by(float r, uint32_t u) {
    float ulp, inv;
    e4m3_step(r, ulp, inv);
    const float q = floorf(fmaf((float)u, 0x1p-20f, r * inv)) * ulp;
    return r > 0.f ? fminf(fmaxf(q, 0x1p-9f), 448.f) : r;
}
// What m may be of its old value, in gradients, to fall by itself.  With beta1 = 0.9 such an m falls by 1/16 or more, which is half of e4m3's largest step:
// only below the normal values does nearest keep it then.
constexpr float FALLS = 0.375f;
// m (new) in units of the scale (im: its inverse), of which the old value was `old`: rounded to nearest by the conversion behind, unless it falls by itself and by
// less than half a step.  There nearest would keep it, for good where the gradient has ended, while the root of v falls on: such an m is rounded down
// or up by 12 random bits, without bias.
__device__ __forceinline__ float let_fall(float m, float old, float b1, float c1, float im, uint32_t u) {
    const float r = fabsf(m) * im, r0 = fabsf(old) * im;
    float ulp, inv;
    e4m3_step(r, ulp, inv);
    const bool alone = fabsf(m - b1 * old) <= FALLS * c1 * fabsf(old);
    const float q = fminf(floorf(fmaf((float)u, 0x1p-12f, r * inv)) * ulp, 448.f);
    return copysignf(alone && r0 - r < 0.5f * ulp ? q : r, m);
}

template <typename P, typename G, bool MASTER, int BITS, bool TAIL>
__device__ __forceinline__ void adamw_block(const AdamArgs& a, const AdamTensor& t, const AdamStep& s, uint32_t key, int64_t i) {
    const int64_t left = t.n - i;
    if (TAIL && left <= -QBLOCK) return;            // the other lanes of a block of scales stay for its maximum
    float g[LANE], w[LANE], m[LANE], v[LANE];
    const int64_t blk = i / QBLOCK;
    float ms = 0.f, vs = 0.f;
    uint2 qm, qv;
    load_lane<G, TAIL>((const G*)t.g + i, left, g);
    if (MASTER) load_lane<float, TAIL>(t.master + i, left, w);
    else load_lane<P, TAIL>((const P*)t.p + i, left, w);
    if constexpr (BITS == 32) {
        load_lane<float, TAIL>((const float*)t.m + i, left, m);
        load_lane<float, TAIL>((const float*)t.v + i, left, v);
    } else {
        qm = load_bytes<TAIL>((const unsigned char*)t.m + i, left);
        qv = load_bytes<TAIL>((const unsigned char*)t.v + i, left);
        if (!TAIL || left > 0) { ms = t.ms[blk]; vs = t.vs[blk]; }
        from_q(qm, ms, m);
        from_q(qv, vs, v);
    }
    const float keep = 1.f - s.lr * t.wd;
    float tm = 0.f, tv = 0.f, fall = -INFINITY;
    unsigned low = ~0u;
    auto moved = [&](float p, float mean, float r) __attribute__((always_inline)) {
        return fmaf(-s.size * mean, __builtin_amdgcn_rcpf(fmaf(r, s.inv_root, a.eps)), p * keep);
    };
#pragma unroll
    for (int e = 0; e < LANE; ++e) {
        if (BITS == 8) v[e] = rounded(v[e], v[e]);
        const float x = rounded(g[e], s.clip), old = fabsf(m[e]);
        m[e] = rounded(a.b1, m[e]) + rounded(a.c1, x);
        // above -(half of the smallest step): let_fall may have something to do
        if (BITS == 8) fall = fmaxf(fall, fminf(fmaf(1.0625f, fabsf(m[e]), -old), fmaf(FALLS, old, -fabsf(x))));
        if (BITS == 8) asm("" : "+v"(fall));
        v[e] = rounded(a.b2, v[e]) + rounded(a.c2, rounded(x, x));
        if (BITS == 32) w[e] = moved(w[e], m[e], root(v[e]));
        else low = min(low, __float_as_uint(v[e]) - 1u);
    }
    if constexpr (BITS == 8) {
        auto update = [&](auto tiny) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < LANE; ++e) {
                v[e] = kept_root<tiny.value>(v[e]);
                w[e] = moved(w[e], m[e], v[e]);
                tm = fmaxf(tm, fabsf(m[e]));            // of what does not exist: zeros
                tv = fmaxf(tv, v[e]);
            }
        };
        if (seldom(low < 0x7FFFFFu)) update(std::true_type{});         // a v below the normal numbers, and not 0
        else update(std::false_type{});
    }
    if (MASTER) store_lane<float, TAIL>(t.master + i, left, w);
    store_lane<P, TAIL>((P*)t.p + i, left, w);
    if constexpr (BITS == 32) {
        store_lane<float, TAIL>((float*)t.m + i, left, m);
        store_lane<float, TAIL>((float*)t.v + i, left, v);
    } else {
        if (seldom(tv == INFINITY)) {       // a square beyond fp32 made an update of 0; its moments stay, or the block's scales would be infinite
            float old[LANE];
            again_from_q(qm, ms, old);
            tm = tv = 0.f;
#pragma unroll
            for (int e = 0; e < LANE; ++e) {
                m[e] = v[e] == INFINITY ? old[e] : m[e];
                tm = fmaxf(tm, fabsf(m[e]));
            }
            __builtin_amdgcn_sched_barrier(0);
            again_from_q(qv, vs, old);
#pragma unroll
            for (int e = 0; e < LANE; ++e) {
                v[e] = v[e] == INFINITY ? old[e] : v[e];
                tv = fmaxf(tv, v[e]);
            }
        }
        tm = block_max(tm);
        tv = block_max(tv);
        const float im = rounded(1.f / tm, 448.f), iv = rounded(1.f / tv, 448.f);
        const uint32_t h = (uint32_t)i * 0x9E3779B1u + (uint32_t)(i >> 32) * 0x27D4EB2Fu + key;
#pragma unroll
        for (int e = 0; e < LANE; ++e) v[e] = round_up_by(rounded(v[e], iv), dither(h + e * 0x9E3779B1u) >> 12);
        store_bytes<TAIL>((unsigned char*)t.v + i, left, to_q(v));
        if (seldom(fall >= tm * (-0x1p-10f / 448.f) && tm > TOP_MIN)) {
            again_from_q(qm, ms, v);        // the old ones
            uint32_t again = h;         // the hashes are made again, rather than held in eight registers
            asm("" : "+v"(again));
#pragma unroll
            for (int e = 0; e < LANE; ++e) {
                m[e] = let_fall(m[e], v[e], a.b1, a.c1, im, dither(again + e * 0x9E3779B1u) & 0xFFFu);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int e = 0; e < LANE; ++e) m[e] *= im;
        }
        store_bytes<TAIL>((unsigned char*)t.m + i, left, to_q(m));
        if constexpr (TAIL) {
            if (threadIdx.x % (QBLOCK / LANE) == 0 && left > 0) {
                t.ms[blk] = tm * (1.f / 448.f);
                t.vs[blk] = tv * (1.f / 448.f);
            }
        } else {
            __shared__ float sc[2][CHUNK / QBLOCK];         // a block's scales are written together: 739 -> 732 us for 218 M elements
            if (threadIdx.x % (QBLOCK / LANE) == 0) {
                sc[0][threadIdx.x / (QBLOCK / LANE)] = tm * (1.f / 448.f);
                sc[1][threadIdx.x / (QBLOCK / LANE)] = tv * (1.f / 448.f);
            }
            __syncthreads();
            if (threadIdx.x < CHUNK / QBLOCK) {
                const int64_t b0 = i / CHUNK * (CHUNK / QBLOCK) + threadIdx.x;
                t.ms[b0] = sc[0][threadIdx.x];
                t.vs[b0] = sc[1][threadIdx.x];
            }
        }
    }
}

// bf16 with fp32 copies and gradients, 32-bit states: 44 M elements, 1.3 GB in 213 to 225 us by box (5.9 to 6.2 TB/s; a copy of 1 GiB reaches 6.2).  8-bit states: 218 M
// elements, 3.9 GB in 704 us (5.6 TB/s).  Four elements a lane with conditions took 236 and 756; eight, and conditions only in a tensor's last block, 223 and 713; copies
// and states past the caches the rest.  A block takes CHUNK elements and ends: with 2, 4, 8 and 16 times as many, 218 (of then) became 233, 240, 252 and 275.
template <typename P, typename G, bool MASTER, int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
    AdamStep s;
    if (!adam_step(a, s)) return;
    int k = 0;
#pragma unroll
    for (int i = 0; i < ADAM_TENSORS; ++i) k += (int)blockIdx.x >= a.end[i];
    const AdamTensor& t = a.t[k];
    const int64_t at = (int64_t)((int)blockIdx.x - (k > 0 ? a.end[k - 1] : 0)) * CHUNK, i = at + threadIdx.x * LANE;
    const uint32_t key = a.seed + 0x85EBCA77u * (uint32_t)(a.first + k + 1) + 0xC2B2AE3Du * s.step;
    if (at + CHUNK <= t.n) adamw_block<P, G, MASTER, BITS, false>(a, t, s, key, i);
    else adamw_block<P, G, MASTER, BITS, true>(a, t, s, key, i);
}

// ---- global norm -----------------------------------------------------------
constexpr int NORM_TENSORS = 160, NORM_BLOCKS = 2048, NORM_CHUNK = 4 * CHUNK;
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

// partial[block]: sum of the squares of the block's chunks, in fp64, where no square overflows.  870 MB of fp32 gradients in 187 us, 4.6 TB/s: what ran ahead
// still has written lines in the last cache.  More blocks, fewer, and shorter chunks are within 2 %.
template <typename G, bool TAIL> __device__ __forceinline__ void add_squares(const G* g, int64_t left, double (&s)[2]) {
    float x[NORM_CHUNK / CHUNK][LANE];
#pragma unroll
    for (int r = 0; r < NORM_CHUNK / CHUNK; ++r) load_lane<G, TAIL>(g + r * CHUNK, left - r * CHUNK, x[r]);
#pragma unroll
    for (int r = 0; r < NORM_CHUNK / CHUNK; ++r)
#pragma unroll
        for (int e = 0; e < LANE; ++e) s[e & 1] = fma((double)x[r][e], (double)x[r][e], s[e & 1]);
}
template <typename G>
__global__ __launch_bounds__(256) void grad_norm_kernel(NormArgs a, double* __restrict__ partial) {
    __shared__ double red[4];
    double s[2] = {0., 0.};
    int k = 0;
    for (int c = blockIdx.x; c < a.end[a.n_tensors - 1]; c += gridDim.x) {
        while (c >= a.end[k]) ++k;
        const int64_t at = (int64_t)(c - (k > 0 ? a.end[k - 1] : 0)) * NORM_CHUNK, i = at + threadIdx.x * LANE, n = a.n[k];
        if (at + NORM_CHUNK <= n) add_squares<G, false>((const G*)a.g[k] + i, n - i, s);
        else add_squares<G, true>((const G*)a.g[k] + i, n - i, s);
    }
    const double t = wave_sum64(s[0] + s[1]);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = t;
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
void adamw_launch(const AdamArgs& a, int grid, hipStream_t st) {
    adamw_kernel<P, G, MASTER, BITS><<<grid, 256, 0, st>>>(a);
}
template <typename P, bool MASTER>
void adamw_dispatch(const AdamArgs& a, int grid, bool g32, bool bits8, hipStream_t st) {
    if (g32) bits8 ? adamw_launch<P, float, MASTER, 8>(a, grid, st) : adamw_launch<P, float, MASTER, 32>(a, grid, st);
    else bits8 ? adamw_launch<P, bf16_t, MASTER, 8>(a, grid, st) : adamw_launch<P, bf16_t, MASTER, 32>(a, grid, st);
}

}  // namespace

extern "C" {

cf_status cf_adamw_step(const cf_adamw_desc* d, const cf_adamw_tensor* tensors, int32_t n_tensors, cf_stream stream) {
    if (!d || (!tensors && n_tensors > 0)) return CF_ERR_NULL;
    for (int dt : {d->p_dtype, d->g_dtype})
        if (dt != CF_BF16 && dt != CF_F32) return CF_ERR_DTYPE;
    if (n_tensors < 0 || (d->state_bits != 8 && d->state_bits != 32)) return CF_ERR_SHAPE;
    if (!(d->lr >= 0.) || !is_finite(d->lr) || !(d->beta1 >= 0. && d->beta1 < 1.) || !(d->beta2 >= 0. && d->beta2 < 1.) || !((float)d->eps >= 0x1p-126f) ||
        !is_finite(d->eps) || !is_finite(d->grad_scale) || (!d->step_dev && d->step < 1))
        return CF_ERR_SHAPE;
    if (d->norm_dev && !(d->max_norm > 0.f)) return CF_ERR_SHAPE;
    if (off(d->norm_dev, 4) || off(d->step_dev, 4) || off(d->lr_dev, 4)) return CF_ERR_SHAPE;
    const bool bits8 = d->state_bits == 8;
    bool master = false, plain = false;
    for (int k = 0; k < n_tensors; ++k) {
        const cf_adamw_tensor& t = tensors[k];
        if (t.n < 0 || t.n > (int64_t)1 << 34 || !is_finite(t.weight_decay) || t.weight_decay < 0.f) return CF_ERR_SHAPE;
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
    a.beta1 = d->beta1; a.beta2 = d->beta2; a.lr = (float)d->lr;
    a.b1 = (float)d->beta1; a.b2 = (float)d->beta2; a.c1 = (float)(1. - d->beta1); a.c2 = (float)(1. - d->beta2);
    a.eps = (float)d->eps; a.step = d->step < 1 ? 1 : d->step; a.seed = d->seed;
    adam_scalars(a.beta1, a.beta2, d->lr, a.step, a.size, a.inv_root);
    a.grad_scale = d->grad_scale; a.max_norm = d->max_norm;
    a.norm_dev = d->norm_dev; a.lr_dev = d->lr_dev; a.step_dev = d->step_dev;
    int k = 0;
    while (k < n_tensors) {
        // as many tensors as the arguments hold and one launch may have blocks, or a single one, whose 2^34 elements at most are 2^23 blocks
        a.first = k;
        int64_t blocks = 0;
        bool full = false;
        for (int i = 0; i < ADAM_TENSORS; ++i) {
            a.end[i] = INT32_MAX;
            if (k >= n_tensors) continue;
            const cf_adamw_tensor& t = tensors[k];
            const int64_t more = (t.n + CHUNK - 1) / CHUNK;
            if (full || (blocks > 0 && blocks + more > MAX_GRID)) { full = true; continue; }
            ++k;
            blocks += more;
            a.t[i] = AdamTensor{t.p, t.master, t.g, t.m, t.v, t.m_scale, t.v_scale, t.n, t.weight_decay};
            a.end[i] = (int32_t)blocks;
        }
        if (blocks == 0) continue;
        if (d->p_dtype == CF_F32) adamw_dispatch<float, false>(a, (int)blocks, d->g_dtype == CF_F32, bits8, st);
        else if (master) adamw_dispatch<bf16_t, true>(a, (int)blocks, d->g_dtype == CF_F32, bits8, st);
        else adamw_dispatch<bf16_t, false>(a, (int)blocks, d->g_dtype == CF_F32, bits8, st);
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
