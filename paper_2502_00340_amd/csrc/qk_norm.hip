// Norm of each query and key head with the rotary rotation in the same pass, forward and backward (on kept rows).
//
// A head of d columns is held by d / (2 VN) neighbouring lanes: each has the VN columns of the lower half from its own on and
// those of the upper half that they are rotated with (two 16-byte loads), so that the rotation stays in a lane and the sums over
// a head are a few steps inside a wave.  A wave takes one row (or several, of few heads) and walks through its heads, so that a
// lane loads its table entries once per row.  HBM-bound: x in and y out, or x, dy in and dx out.
#include "common.h"

namespace cf {

// what a lane holds of a head: VN columns of the lower and VN of the upper half, as they are stored and widened
template <typename T> struct Half2 {
    static constexpr int VN = Vec<T>::N;
    float lo[VN], hi[VN];
    __device__ __forceinline__ void store(T* p, int half) const {
        Vec<T>::store(p, lo);
        Vec<T>::store(p + half, hi);
    }
};
typedef unsigned u32x4q __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void widen16(const u32x4q& b, float (&o)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(b[i]);
}
__device__ __forceinline__ void widen16(const u32x4q& b, float (&o)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[2 * i] = __uint_as_float(b[i] << 16);
        o[2 * i + 1] = __uint_as_float(b[i] & 0xFFFF0000u);
    }
}
template <typename T> struct Raw2 {
    u32x4q lo, hi;
    __device__ __forceinline__ void load(const T* p, int half) {
        lo = *reinterpret_cast<const u32x4q*>(p);
        hi = *reinterpret_cast<const u32x4q*>(p + half);
    }
    __device__ __forceinline__ Half2<T> wide() const {
        Half2<T> h;
        widen16(lo, h.lo);
        widen16(hi, h.hi);
        return h;
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
    int64_t first;          // row of the launch's first block
};

template <typename T, int LANES> struct RowTables {
    static constexpr int VN = Vec<T>::N, HALF = VN * LANES;
    float c[VN], s[VN];
    __device__ __forceinline__ void load(const QkShape& sh, int64_t row, int part) {
        u32x4q a[VN / 4], b[VN / 4];
#pragma unroll
        for (int q = 0; q < VN / 4; ++q) {
            a[q] = u32x4q{0x3F800000u, 0x3F800000u, 0x3F800000u, 0x3F800000u};      // no tables: no rotation
            b[q] = u32x4q{0u, 0u, 0u, 0u};
        }
        if (sh.cos != nullptr) {
            const int at = sh.positions != nullptr ? sh.positions[row] : (int)(row % sh.S), pos = min(max(at, 0), sh.S - 1);
            const int64_t i = (int64_t)pos * HALF + part * VN;
#pragma unroll
            for (int q = 0; q < VN / 4; ++q) {
                a[q] = reinterpret_cast<const u32x4q*>(sh.cos + i)[q];
                b[q] = reinterpret_cast<const u32x4q*>(sh.sin + i)[q];
            }
        }
#pragma unroll
        for (int e = 0; e < VN; ++e) {
            c[e] = __uint_as_float(a[e / 4][e % 4]);
            s[e] = __uint_as_float(b[e / 4][e % 4]);
        }
    }
};

template <typename T> struct QkPtr {
    T *q, *k;
    int64_t qs, ks;
};

// Heads h0, h0 + hp, ... of H, U at a time: all loads of U heads ahead of the arithmetic.  A lane group that has no head left does what the one
// with the last head does, so that no access hangs on a branch; in place too, since the last head belongs to the last U.
constexpr int QK_U = 4;

// 8192 rows of 32 + 8 heads of 128 in bf16: 168 MB in 30.0 us, 5.6 TB/s (a copy of 1 GiB reaches 6.2); one head at a time 33.5.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void qk_norm_fwd_kernel(QkShape sh, QkPtr<const T> in, QkPtr<T> out, int n_rows) {
    constexpr int VN = Vec<T>::N, HALF = VN * LANES, D = 2 * HALF, GROUPS = 64 / LANES;
    const int lane = threadIdx.x & 63, part = lane & (LANES - 1), group = lane / LANES;
    const int h0 = group & (sh.hp - 1), rpw = GROUPS / sh.hp;
    const int64_t row = sh.first + ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * rpw + group / sh.hp;
    if (row >= n_rows) return;
    RowTables<T, LANES> tab;
    tab.load(sh, row, part);
    auto heads = [&](const T* src, T* dst, int H, const void* gain) __attribute__((always_inline)) {
        Raw2<T> graw;
        graw.load((const T*)gain + part * VN, HALF);
        for (int hb = 0; hb < H; hb += QK_U * sh.hp) {
            Raw2<T> x[QK_U];
#pragma unroll
            for (int u = 0; u < QK_U; ++u) x[u].load(src + (int64_t)min(hb + u * sh.hp + h0, H - 1) * D + part * VN, HALF);
            const Half2<T> g = graw.wide();
#pragma unroll
            for (int u = 0; u < QK_U; ++u) {
                if (u > 0 && hb + u * sh.hp >= H) break;
                const Half2<T> w = x[u].wide();
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < VN; ++e) ss += w.lo[e] * w.lo[e] + w.hi[e] * w.hi[e];
                const float rstd = rsqrtf(lanes_sum<LANES>(ss) * (1.0f / D) + sh.eps);
                Half2<T> y;
#pragma unroll
                for (int e = 0; e < VN; ++e) {
                    const float a = w.lo[e] * rstd * g.lo[e], b = w.hi[e] * rstd * g.hi[e];
                    y.lo[e] = a * tab.c[e] - b * tab.s[e];
                    y.hi[e] = b * tab.c[e] + a * tab.s[e];
                }
                y.store(dst + (int64_t)min(hb + u * sh.hp + h0, H - 1) * D + part * VN, HALF);
                __builtin_amdgcn_sched_barrier(0);          // one head after the other: waves hide the latencies, and registers decide how many there are
            }
        }
    };
    heads(in.q + row * in.qs, out.q + row * out.qs, sh.Hq, sh.gq);
    heads(in.k + row * in.ks, out.k + row * out.ks, sh.Hkv, sh.gk);
}

// Blocks that the live rows are dealt out to, and so the partials of the gain gradients: a function of the live rows alone.
constexpr int QK_BWD_BLOCKS = 768;
__host__ __device__ inline int qk_bwd_nblk(int n_rows) {
    const int b = (n_rows + 3) / 4;
    return b < QK_BWD_BLOCKS ? b : QK_BWD_BLOCKS;
}

// partial [nblk][2][D]: the block's sums of u*n over its rows, of the query heads and of the key heads (null: not wanted).
// Of dy rotated back (u), dx = rstd (u*g - n mean(u*g*n)).  4096 kept of 8192 rows of 32 + 8 heads of 128 in bf16: 127 MB in 24.2 us, 5.3 TB/s, with
// two heads' loads ahead and the lanes' gain sums by way of LDS; one head at a time and sums across lanes 32.5.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void qk_norm_bwd_kernel(QkShape sh, QkPtr<const T> in, QkPtr<const T> dy, const int32_t* __restrict__ idx,
                                                          int n_max, const int32_t* __restrict__ n_dev, QkPtr<T> dx,
                                                          float* __restrict__ partial) {
    constexpr int VN = Vec<T>::N, HALF = VN * LANES, D = 2 * HALF, GROUPS = 64 / LANES, U = 2;
    __shared__ float red[4 * GROUPS * D];
    const int n_rows = live_rows(n_max, n_dev), nblk = qk_bwd_nblk(n_rows);
    if ((int)blockIdx.x >= nblk) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane & (LANES - 1), group = lane / LANES;
    const int h0 = group & (sh.hp - 1), rpw = GROUPS / sh.hp;
    float acc[2][2 * VN];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 2 * VN; ++e) acc[k][e] = 0.f;
    for (int64_t j = ((int64_t)blockIdx.x * 4 + wave) * rpw + group / sh.hp; j < n_rows; j += (int64_t)nblk * 4 * rpw) {
        const int64_t row = idx != nullptr ? idx[j] : j;
        RowTables<T, LANES> tab;
        tab.load(sh, row, part);
        auto heads = [&](const T* xs, const T* ys, T* dst, int H, const void* gain, float (&ac)[2 * VN]) __attribute__((always_inline)) {
            Raw2<T> graw;
            graw.load((const T*)gain + part * VN, HALF);
            for (int hb = 0; hb < H; hb += U * sh.hp) {
                Raw2<T> x[U], y[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t at = (int64_t)min(hb + u * sh.hp + h0, H - 1) * D + part * VN;
                    x[u].load(xs + at, HALF);
                    y[u].load(ys + at, HALF);
                }
                const Half2<T> g = graw.wide();
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (u > 0 && hb + u * sh.hp >= H) break;
                    const float mine = hb + u * sh.hp + h0 < H ? 1.f : 0.f;         // a head that is another group's does not count twice
                    const Half2<T> w = x[u].wide();
                    Half2<T> v = y[u].wide();
                    float ss = 0.f, sd = 0.f;
#pragma unroll
                    for (int e = 0; e < VN; ++e) {      // u = R^T dy in place of dy
                        const float a = v.lo[e] * tab.c[e] + v.hi[e] * tab.s[e], b = v.hi[e] * tab.c[e] - v.lo[e] * tab.s[e];
                        v.lo[e] = a; v.hi[e] = b;
                        ss += w.lo[e] * w.lo[e] + w.hi[e] * w.hi[e];
                        sd += a * g.lo[e] * w.lo[e] + b * g.hi[e] * w.hi[e];
                    }
                    const float rstd = rsqrtf(lanes_sum<LANES>(ss) * (1.0f / D) + sh.eps);
                    const float c = lanes_sum<LANES>(sd) * rstd * (1.0f / D);      // mean(u*g*n)
                    const float rm = rstd * mine;
#pragma unroll
                    for (int e = 0; e < VN; ++e) {
                        ac[e] += v.lo[e] * (w.lo[e] * rm);
                        ac[VN + e] += v.hi[e] * (w.hi[e] * rm);
                        v.lo[e] = rstd * (v.lo[e] * g.lo[e] - w.lo[e] * rstd * c);
                        v.hi[e] = rstd * (v.hi[e] * g.hi[e] - w.hi[e] * rstd * c);
                    }
                    v.store(dst + (int64_t)min(hb + u * sh.hp + h0, H - 1) * D + part * VN, HALF);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        heads(in.q + row * in.qs, dy.q + j * dy.qs, dx.q + j * dx.qs, sh.Hq, sh.gq, acc[0]);
        heads(in.k + row * in.ks, dy.k + j * dy.ks, dx.k + j * dx.ks, sh.Hkv, sh.gk, acc[1]);
    }
    if (partial == nullptr) return;
    // the lane groups' sums by way of LDS, the queries' and then the keys': all threads add up rows of it, then a thread a column their sums
    constexpr int SUB = 256 / D;
    const int col = threadIdx.x % D, sub = threadIdx.x / D;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (k > 0) __syncthreads();
        float* mine = red + (wave * GROUPS + group) * D;
#pragma unroll
        for (int e = 0; e < VN; ++e) {
            mine[part * VN + e] = acc[k][e];
            mine[HALF + part * VN + e] = acc[k][VN + e];
        }
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < 4 * GROUPS / SUB; ++r) s += red[(sub + r * SUB) * D + col];
        if (SUB > 1) {
            __syncthreads();
            red[threadIdx.x] = s;
            __syncthreads();
            s = 0.f;
#pragma unroll
            for (int r = 0; r < SUB; ++r) s += red[r * D + col];
        }
        if (threadIdx.x < D) partial[(int64_t)blockIdx.x * (2 * D) + k * D + col] = s;
    }
}

// dg[c] (+)= sum over the blocks' partials: 16 columns a block, 64 row groups, all of a thread's loads in flight at once.  4 us, those of a launch.
template <typename T, bool ACC>
__global__ __launch_bounds__(1024) void qk_gain_kernel(const float* __restrict__ partial, int n_max, const int32_t* __restrict__ n_dev,
                                                       int d, T* __restrict__ dgq, T* __restrict__ dgk) {
    __shared__ float red[64][17];
    const int nblk = qk_bwd_nblk(live_rows(n_max, n_dev));
    const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < QK_BWD_BLOCKS / 64; ++i) s += rg + 64 * i < nblk ? partial[(int64_t)(rg + 64 * i) * (2 * d) + c] : 0.f;
    red[rg][cl] = s;
    __syncthreads();
    if (threadIdx.x < 16) {
        float t = 0.f;
#pragma unroll
        for (int r = 0; r < 64; ++r) t += red[r][threadIdx.x];
        T* out = c < d ? dgq + c : dgk + (c - d);
        if (ACC) *out += from_f32<T>(t);
        else *out = from_f32<T>(t);
    }
}

// ---------------------------------------------------------------------------

static QkShape qk_shape(const cf_layer_desc& L, const cf_qk_norm& p, int groups) {
    int hp = 1;
    while (hp < groups && hp < L.Hq + L.Hkv) hp *= 2;
    return QkShape{L.Hq, L.Hkv, L.S, hp, L.rms_eps, p.gq, p.gk, p.rope_cos, p.rope_sin, p.positions, 0};
}

template <typename T, typename U> static QkPtr<T> qk_ptr(const U& t, const cf_layer_desc& L) {
    return QkPtr<T>{(T*)t.q, (T*)t.k, t.q_stride ? t.q_stride : (int64_t)L.Hq * L.d, t.k_stride ? t.k_stride : (int64_t)L.Hkv * L.d};
}

template <typename T, int LANES>
static void qk_fwd_t(const cf_layer_desc& L, const cf_qk_norm& p, const cf_qk& in, int n_rows, const cf_qk& out, hipStream_t st) {
    QkShape sh = qk_shape(L, p, 64 / LANES);
    const int rows_per_block = 4 * (64 / LANES / sh.hp);
    for (; sh.first < n_rows; sh.first += (int64_t)MAX_GRID * rows_per_block) {
        const int64_t left = n_rows - sh.first, blocks = (left + rows_per_block - 1) / rows_per_block;
        qk_norm_fwd_kernel<T, LANES><<<(int)(blocks < MAX_GRID ? blocks : MAX_GRID), 256, 0, st>>>(sh, qk_ptr<const T>(in, L), qk_ptr<T>(out, L), n_rows);
    }
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
        const int grid = 2 * L.d / 16;
        if (acc_f32) qk_gain_kernel<float, true><<<grid, 1024, 0, st>>>(partial, rows.n, rows.dev, L.d, (float*)dgq, (float*)dgk);
        else if (L.dtype == CF_F32) qk_gain_kernel<float, false><<<grid, 1024, 0, st>>>(partial, rows.n, rows.dev, L.d, (float*)dgq, (float*)dgk);
        else qk_gain_kernel<bf16_t, false><<<grid, 1024, 0, st>>>(partial, rows.n, rows.dev, L.d, (bf16_t*)dgq, (bf16_t*)dgk);
    }
    return hipGetLastError();
}

}  // namespace cf
