// Norm of each query and key head with the rotary rotation in the same pass, forward and backward (on kept rows).
//
// A head of d columns is held by d / (2 VN) neighbouring lanes: each has the VN columns of the lower half from its own on and
// those of the upper half that they are rotated with (two 16-byte loads), so that the rotation stays in a lane and the sums over
// a head are a few steps inside a wave.  A wave takes one row (or several, of few heads) and walks through its heads, so that a
// lane loads its table entries once per row.  HBM-bound: x in and y out, or x, dy in and dx out.
#include "common.h"

namespace cf {

// what a lane holds of a head: VN columns of the lower and VN of the upper half
template <typename T> struct Half2 {
    static constexpr int VN = Vec<T>::N;
    float lo[VN], hi[VN];
    __device__ __forceinline__ void load(const T* p, int half) {
        Vec<T>::load(p, lo);
        Vec<T>::load(p + half, hi);
    }
    __device__ __forceinline__ void store(T* p, int half) const {
        Vec<T>::store(p, lo);
        Vec<T>::store(p + half, hi);
    }
};

template <int LANES> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = LANES >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// How a wave's lane groups are dealt out to rows and heads: hp groups (a power of two) per row
struct QkShape {
    int Hq, Hkv, S;
    int hp;                 // groups that share a row
    float eps;
    const void *gq, *gk;
    const float *cos, *sin;
    const int32_t* positions;
};

template <typename T, int LANES> struct RowTables {
    static constexpr int VN = Vec<T>::N, HALF = VN * LANES;
    float c[VN], s[VN];
    __device__ __forceinline__ void load(const QkShape& sh, int64_t row, int part) {
        if (sh.cos == nullptr) {
#pragma unroll
            for (int e = 0; e < VN; ++e) { c[e] = 1.f; s[e] = 0.f; }
            return;
        }
        int pos = sh.positions != nullptr ? sh.positions[row] : (int)(row % sh.S);
        pos = pos < 0 ? 0 : (pos < sh.S ? pos : sh.S - 1);
        const int64_t at = (int64_t)pos * HALF + part * VN;
#pragma unroll
        for (int q = 0; q < VN / 4; ++q) {
            const float4 a = reinterpret_cast<const float4*>(sh.cos + at)[q], b = reinterpret_cast<const float4*>(sh.sin + at)[q];
            c[4 * q] = a.x; c[4 * q + 1] = a.y; c[4 * q + 2] = a.z; c[4 * q + 3] = a.w;
            s[4 * q] = b.x; s[4 * q + 1] = b.y; s[4 * q + 2] = b.z; s[4 * q + 3] = b.w;
        }
    }
};

template <typename T> struct QkPtr {
    T *q, *k;
    int64_t qs, ks;
    __device__ __forceinline__ T* head(int64_t row, int h, int Hq, int d) const {
        return h < Hq ? q + row * qs + (int64_t)h * d : k + row * ks + (int64_t)(h - Hq) * d;
    }
};

template <typename T, int LANES>
__global__ __launch_bounds__(256) void qk_norm_fwd_kernel(QkShape sh, QkPtr<const T> in, QkPtr<T> out, int n_rows) {
    constexpr int VN = Vec<T>::N, HALF = VN * LANES, D = 2 * HALF, GROUPS = 64 / LANES;
    const int lane = threadIdx.x & 63, part = lane & (LANES - 1), group = lane / LANES;
    const int h0 = group & (sh.hp - 1), rpw = GROUPS / sh.hp;
    const int64_t row = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * rpw + group / sh.hp;
    if (row >= n_rows) return;
    const int heads = sh.Hq + sh.Hkv;
    RowTables<T, LANES> tab;
    tab.load(sh, row, part);
    for (int h = h0; h < heads; h += sh.hp) {
        Half2<T> x, g, y;
        x.load(in.head(row, h, sh.Hq, D) + part * VN, HALF);
        g.load((const T*)(h < sh.Hq ? sh.gq : sh.gk) + part * VN, HALF);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VN; ++e) ss += x.lo[e] * x.lo[e] + x.hi[e] * x.hi[e];
        const float rstd = rsqrtf(lanes_sum<LANES>(ss) * (1.0f / D) + sh.eps);
#pragma unroll
        for (int e = 0; e < VN; ++e) {
            const float a = x.lo[e] * rstd * g.lo[e], b = x.hi[e] * rstd * g.hi[e];
            y.lo[e] = a * tab.c[e] - b * tab.s[e];
            y.hi[e] = b * tab.c[e] + a * tab.s[e];
        }
        y.store(out.head(row, h, sh.Hq, D) + part * VN, HALF);
    }
}

// Blocks that the live rows are dealt out to, and so the partials of the gain gradients: a function of the live rows alone.
__host__ __device__ inline int qk_bwd_nblk(int n_rows) {
    const int b = (n_rows + 3) / 4;
    return b < 1024 ? b : 1024;
}

// partial [nblk][2][D]: the block's sums of u*n over its rows, of the query heads and of the key heads (null: not wanted).
template <typename T, int LANES>
__global__ __launch_bounds__(256) void qk_norm_bwd_kernel(QkShape sh, QkPtr<const T> in, QkPtr<const T> dy, const int32_t* __restrict__ idx,
                                                          int n_max, const int32_t* __restrict__ n_dev, QkPtr<T> dx,
                                                          float* __restrict__ partial) {
    constexpr int VN = Vec<T>::N, HALF = VN * LANES, D = 2 * HALF, GROUPS = 64 / LANES;
    __shared__ float red[4][2 * D];
    const int n_rows = live_rows(n_max, n_dev), nblk = qk_bwd_nblk(n_rows);
    if ((int)blockIdx.x >= nblk) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane & (LANES - 1), group = lane / LANES;
    const int h0 = group & (sh.hp - 1), rpw = GROUPS / sh.hp;
    const int heads = sh.Hq + sh.Hkv;
    float acc[2][2][VN];
#pragma unroll
    for (int i = 0; i < 4 * VN; ++i) (&acc[0][0][0])[i] = 0.f;
    for (int64_t j = ((int64_t)blockIdx.x * 4 + wave) * rpw + group / sh.hp; j < n_rows; j += (int64_t)nblk * 4 * rpw) {
        const int64_t row = idx != nullptr ? idx[j] : j;
        RowTables<T, LANES> tab;
        tab.load(sh, row, part);
        for (int h = h0; h < heads; h += sh.hp) {
            const bool is_q = h < sh.Hq;
            Half2<T> x, y, g;
            x.load(in.head(row, h, sh.Hq, D) + part * VN, HALF);
            y.load(dy.head(j, h, sh.Hq, D) + part * VN, HALF);
            g.load((const T*)(is_q ? sh.gq : sh.gk) + part * VN, HALF);
            float ss = 0.f, sd = 0.f;
#pragma unroll
            for (int e = 0; e < VN; ++e) {      // u = R^T dy in place of dy
                const float a = y.lo[e] * tab.c[e] + y.hi[e] * tab.s[e], b = y.hi[e] * tab.c[e] - y.lo[e] * tab.s[e];
                y.lo[e] = a; y.hi[e] = b;
                ss += x.lo[e] * x.lo[e] + x.hi[e] * x.hi[e];
                sd += a * g.lo[e] * x.lo[e] + b * g.hi[e] * x.hi[e];
            }
            const float rstd = rsqrtf(lanes_sum<LANES>(ss) * (1.0f / D) + sh.eps);
            const float c = lanes_sum<LANES>(sd) * rstd * (1.0f / D);      // mean(u*g*n)
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                const float nl = x.lo[e] * rstd, nh = x.hi[e] * rstd;
                const float al = y.lo[e] * nl, ah = y.hi[e] * nh;
                acc[0][0][e] += is_q ? al : 0.f; acc[0][1][e] += is_q ? ah : 0.f;
                acc[1][0][e] += is_q ? 0.f : al; acc[1][1][e] += is_q ? 0.f : ah;
                y.lo[e] = rstd * (y.lo[e] * g.lo[e] - nl * c);
                y.hi[e] = rstd * (y.hi[e] * g.hi[e] - nh * c);
            }
            y.store(dx.head(j, h, sh.Hq, D) + part * VN, HALF);
        }
    }
    if (partial == nullptr) return;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                float v = acc[k][p][e];
#pragma unroll
                for (int o = LANES; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
                if (group == 0) red[wave][k * D + p * HALF + part * VN + e] = v;
            }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * D; c += 256)
        partial[(int64_t)blockIdx.x * (2 * D) + c] = red[0][c] + red[1][c] + red[2][c] + red[3][c];
}

// dg[c] (+)= sum over the blocks' partials: 8 columns a block, 32 row groups
template <typename T, bool ACC>
__global__ __launch_bounds__(256) void qk_gain_kernel(const float* __restrict__ partial, int n_max, const int32_t* __restrict__ n_dev,
                                                      int d, T* __restrict__ dgq, T* __restrict__ dgk) {
    __shared__ float red[32][9];
    const int nblk = qk_bwd_nblk(live_rows(n_max, n_dev));
    const int cl = threadIdx.x & 7, rg = threadIdx.x >> 3, c = blockIdx.x * 8 + cl;
    float s = 0.f;
#pragma unroll 8
    for (int b = rg; b < nblk; b += 32) s += partial[(int64_t)b * (2 * d) + c];
    red[rg][cl] = s;
    __syncthreads();
    if (threadIdx.x < 8) {
        float t = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) t += red[r][threadIdx.x];
        T* out = c < d ? dgq + c : dgk + (c - d);
        if (ACC) *out += from_f32<T>(t);
        else *out = from_f32<T>(t);
    }
}

// ---------------------------------------------------------------------------

static QkShape qk_shape(const cf_layer_desc& L, const cf_qk_norm& p, int groups) {
    int hp = 1;
    while (hp < groups && hp < L.Hq + L.Hkv) hp *= 2;
    return QkShape{L.Hq, L.Hkv, L.S, hp, L.rms_eps, p.gq, p.gk, p.rope_cos, p.rope_sin, p.positions};
}

template <typename T, typename U> static QkPtr<T> qk_ptr(const U& t, const cf_layer_desc& L) {
    return QkPtr<T>{(T*)t.q, (T*)t.k, t.q_stride ? t.q_stride : (int64_t)L.Hq * L.d, t.k_stride ? t.k_stride : (int64_t)L.Hkv * L.d};
}

template <typename T, int LANES>
static void qk_fwd_t(const cf_layer_desc& L, const cf_qk_norm& p, const cf_qk& in, int n_rows, const cf_qk& out, hipStream_t st) {
    const QkShape sh = qk_shape(L, p, 64 / LANES);
    const int rows_per_block = 4 * (64 / LANES / sh.hp);
    qk_norm_fwd_kernel<T, LANES><<<ceil_div(n_rows, rows_per_block), 256, 0, st>>>(sh, qk_ptr<const T>(in, L), qk_ptr<T>(out, L), n_rows);
}

template <typename T, int LANES>
static void qk_bwd_t(const cf_layer_desc& L, const cf_qk_norm& p, const cf_qk& in, const cf_qk& dy, const int32_t* idx, RowCount rows,
                     const cf_qk& dx, float* partial, hipStream_t st) {
    qk_norm_bwd_kernel<T, LANES><<<qk_bwd_nblk(rows.n), 256, 0, st>>>(qk_shape(L, p, 64 / LANES), qk_ptr<const T>(in, L), qk_ptr<const T>(dy, L), idx,
                                                                      rows.n, rows.dev, qk_ptr<T>(dx, L), partial);
}

#define CF_QK_LANES(FN, ...)                                                  \
    switch (L.d / (L.dtype == CF_F32 ? 8 : 16)) {                             \
        case 1: L.dtype == CF_F32 ? FN<float, 1>(__VA_ARGS__) : FN<bf16_t, 1>(__VA_ARGS__); break;     \
        case 2: L.dtype == CF_F32 ? FN<float, 2>(__VA_ARGS__) : FN<bf16_t, 2>(__VA_ARGS__); break;     \
        case 4: L.dtype == CF_F32 ? FN<float, 4>(__VA_ARGS__) : FN<bf16_t, 4>(__VA_ARGS__); break;     \
        case 8: L.dtype == CF_F32 ? FN<float, 8>(__VA_ARGS__) : FN<bf16_t, 8>(__VA_ARGS__); break;     \
        case 16: L.dtype == CF_F32 ? FN<float, 16>(__VA_ARGS__) : FN<bf16_t, 16>(__VA_ARGS__); break;  \
        case 32: FN<float, 32>(__VA_ARGS__); break;                           \
        default: return hipErrorInvalidValue;                                 \
    }

hipError_t launch_qk_norm_fwd(const cf_layer_desc& L, const cf_qk_norm& p, const cf_qk& in, int n_rows, const cf_qk& out, hipStream_t st) {
    if (n_rows <= 0) return hipSuccess;
    CF_QK_LANES(qk_fwd_t, L, p, in, n_rows, out, st)
    return hipGetLastError();
}

size_t qk_norm_partial_bytes(int d, int n_rows) { return (size_t)qk_bwd_nblk(n_rows > 0 ? n_rows : 1) * 2 * d * sizeof(float); }

hipError_t launch_qk_norm_bwd(const cf_layer_desc& L, const cf_qk_norm& p, const cf_qk& in, const cf_qk& dy, const int32_t* idx,
                              RowCount rows, const cf_qk& dx, void* dgq, void* dgk, bool acc_f32, float* partial, hipStream_t st) {
    if (rows.n > 0) {
        float* const into = dgq ? partial : nullptr;
        CF_QK_LANES(qk_bwd_t, L, p, in, dy, idx, rows, dx, into, st)
    }
    if (dgq) {      // no rows: no partials, zeros
        const int grid = 2 * L.d / 8;
        if (acc_f32) qk_gain_kernel<float, true><<<grid, 256, 0, st>>>(partial, rows.n, rows.dev, L.d, (float*)dgq, (float*)dgk);
        else if (L.dtype == CF_F32) qk_gain_kernel<float, false><<<grid, 256, 0, st>>>(partial, rows.n, rows.dev, L.d, (float*)dgq, (float*)dgk);
        else qk_gain_kernel<bf16_t, false><<<grid, 256, 0, st>>>(partial, rows.n, rows.dev, L.d, (bf16_t*)dgq, (bf16_t*)dgk);
    }
    return hipGetLastError();
}

}  // namespace cf
