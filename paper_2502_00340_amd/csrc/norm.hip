// The norm of rows, forward and backward: root mean square (mu = 0) or layer norm,
//   n = (x - mu) * rstd,  rstd = (mean((x - mu)^2) + eps)^(-1/2),  y = n * g + b
//   u = dy * g,  dx = rstd * (u - [layer] mean(u) - n * mean(u * n)),  dg = sum over rows of dy * n,  db = sum of dy
// HBM-bound: rows in, rows out; a row stays in registers from its statistics to its output, and the next row is asked for ahead of them.  The statistics are
// centred sums (the mean first), in fp32: no difference of two large sums.  4096 rows of 4096 bf16 through an index: forward 11.6 us, 5.8 TB/s, backward 19.5, 5.1 TB/s, and 4 for
// the gains' second launch.
#include "common.h"
#include "mfma_util.h"

namespace cf {

struct RowNormArgs {
    const void *x, *g, *b, *dy;
    const int32_t *idx, *n_dev;
    int n_max, H;
    float eps;
    void* out;              // y, or dx
    float *pg, *pb;         // backward: [blocks, H] sums of each block (nullable: frozen gains; pb with b only)
    int blocks;             // most that walk through the rows
};

// Sums of K values over the NT threads that share a row (64: a wave; else the whole block of NT).  `red` holds K * NT / 64 values of one call; calls in turn use
// two of them, so that one barrier a call is enough.
template <int NT, int K> __device__ __forceinline__ void row_sum(float (&v)[K], float* red) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
    if constexpr (NT > 64) {
        constexpr int W = NT / 64;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) red[k * W + (threadIdx.x >> 6)] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) v[k] += red[k * W + w];
        }
    }
}

template <typename T> __device__ __forceinline__ void unpack(const u32x4_t& w, float (&o)[Vec<T>::N]) {
    Vec<T>::load(reinterpret_cast<const T*>(&w), o);
}

// NT threads a row, NV vectors of 16 bytes a thread; blocks of 256 (or NT) threads, so that NT = 64 has four rows a block at a time
template <typename T, int NT, int NV, bool LAYER>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_fwd_kernel(RowNormArgs a) {
    constexpr int VN = Vec<T>::N, BT = NT < 256 ? 256 : NT, RPB = BT / NT;
    __shared__ float red[2][NT > 64 ? NT / 64 : 1];
    const int n_rows = live_rows(a.n_max, a.n_dev), H = a.H, vpr = H / VN, tid = threadIdx.x % NT;
    const float inv_h = 1.f / (float)H;
    const T *g = (const T*)a.g, *b = (const T*)a.b;
    const int64_t step = (int64_t)gridDim.x * RPB;
    int64_t j = (int64_t)blockIdx.x * RPB + threadIdx.x / NT;
    u32x4_t x[NV];
    auto fetch = [&](int64_t j) __attribute__((always_inline)) {
        j = j < n_rows ? j : n_rows - 1;
        const T* row = (const T*)a.x + (a.idx != nullptr ? (int64_t)a.idx[j] : j) * H;
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = *reinterpret_cast<const u32x4_t*>(row + min(tid + i * NT, vpr - 1) * VN);
    };
    if (n_rows == 0) return;
    fetch(j);
    // gains and biases: once a thread
    u32x4_t gv[NV], bv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = tid + i * NT;
        gv[i] = bv[i] = u32x4_t{0u, 0u, 0u, 0u};
        if (v < vpr) {
            gv[i] = *reinterpret_cast<const u32x4_t*>(g + v * VN);
            if (b != nullptr) bv[i] = *reinterpret_cast<const u32x4_t*>(b + v * VN);
        }
    }
    for (; j < n_rows; j += step) {
        float xf[NV][VN], mu = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) unpack<T>(tid + i * NT < vpr ? x[i] : u32x4_t{0u, 0u, 0u, 0u}, xf[i]);
        fetch(j + step);
        if (LAYER) {
            float s[1] = {0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VN; ++e) s[0] += xf[i][e];
            row_sum<NT>(s, red[0]);
            mu = s[0] * inv_h;
        }
        float q[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool have = tid + i * NT < vpr;
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                xf[i][e] = LAYER && !have ? 0.f : xf[i][e] - mu;
                q[0] = fmaf(xf[i][e], xf[i][e], q[0]);
            }
        }
        row_sum<NT>(q, red[1]);
        const float rstd = rsqrtf(fmaf(q[0], inv_h, a.eps));
        T* y = (T*)a.out + j * H;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * NT;
            if (v >= vpr) continue;
            float gf[VN], bf[VN], o[VN];
            unpack<T>(gv[i], gf);
            unpack<T>(bv[i], bf);
#pragma unroll
            for (int e = 0; e < VN; ++e) o[e] = fmaf(xf[i][e] * rstd, gf[e], bf[e]);
            Vec<T>::store(y + v * VN, o);
        }
        if (NT > 64 && !LAYER) __syncthreads();         // red[1] is written again without a barrier in between
    }
}

// Rows that a block of the backward walks through: dealt out evenly, and a function of the live rows, so that the sums' order is one of the sizes.
__host__ __device__ inline int norm_bwd_used(int n_rows, int rpb, int blocks) {
    const int need = (n_rows + rpb - 1) / rpb;
    return need < blocks ? need : blocks;
}

template <typename T, int NT, int NV, bool LAYER>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_bwd_kernel(RowNormArgs a) {
    constexpr int VN = Vec<T>::N, BT = NT < 256 ? 256 : NT, RPB = BT / NT, W = NT > 64 ? NT / 64 : 1;
    __shared__ float red[2][3 * W];
    const int n_rows = live_rows(a.n_max, a.n_dev), H = a.H, vpr = H / VN, tid = threadIdx.x % NT;
    const int used = norm_bwd_used(n_rows, RPB, a.blocks);
    if ((int)blockIdx.x >= used) return;
    const float inv_h = 1.f / (float)H;
    const int64_t step = (int64_t)used * RPB;
    // rows whose loads are in flight beside the one in work; behind the last one it is read again: no load is conditional, or the one waited for would be the last
    constexpr int AHEAD = NV <= 2 ? 2 : 1;
    u32x4_t x[AHEAD][NV], dy[AHEAD][NV], gv[NV];
    float sg[NV][VN], sb[LAYER ? NV : 1][VN];
    auto fetch = [&](u32x4_t (&xr)[NV], u32x4_t (&dr)[NV], int64_t j) __attribute__((always_inline)) {
        j = j < n_rows ? j : n_rows - 1;
        const T* row = (const T*)a.x + (a.idx != nullptr ? (int64_t)a.idx[j] : j) * H;
        const T* drow = (const T*)a.dy + j * H;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = min(tid + i * NT, vpr - 1);
            xr[i] = *reinterpret_cast<const u32x4_t*>(row + v * VN);
            dr[i] = *reinterpret_cast<const u32x4_t*>(drow + v * VN);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * RPB + threadIdx.x / NT;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) fetch(x[k], dy[k], first + k * step);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = tid + i * NT;
        gv[i] = u32x4_t{0u, 0u, 0u, 0u};
        if (v < vpr) gv[i] = *reinterpret_cast<const u32x4_t*>((const T*)a.g + v * VN);
#pragma unroll
        for (int e = 0; e < VN; ++e) {
            sg[i][e] = 0.f;
            if (LAYER) sb[i][e] = 0.f;
        }
    }
    auto take = [&](u32x4_t (&xr)[NV], u32x4_t (&dr)[NV], int64_t j) __attribute__((always_inline)) {
        float xf[NV][VN], df[NV][VN], mu = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool have = tid + i * NT < vpr;
            unpack<T>(have ? xr[i] : u32x4_t{0u, 0u, 0u, 0u}, xf[i]);
            unpack<T>(have ? dr[i] : u32x4_t{0u, 0u, 0u, 0u}, df[i]);
        }
        fetch(xr, dr, j + AHEAD * step);
        if (LAYER) {
            float s[1] = {0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VN; ++e) s[0] += xf[i][e];
            row_sum<NT>(s, red[0]);
            mu = s[0] * inv_h;
        }
        // sums of (x - mu)^2, u * (x - mu) and u
        float s[LAYER ? 3 : 2] = {};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool have = tid + i * NT < vpr;
            float gf[VN];
            unpack<T>(gv[i], gf);
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                xf[i][e] = LAYER && !have ? 0.f : xf[i][e] - mu;
                const float u = df[i][e] * gf[e];
                s[0] = fmaf(xf[i][e], xf[i][e], s[0]);
                s[1] = fmaf(u, xf[i][e], s[1]);
                if constexpr (LAYER) s[2] += u;
            }
        }
        row_sum<NT>(s, red[1]);
        const float rstd = rsqrtf(fmaf(s[0], inv_h, a.eps));
        const float c = s[1] * inv_h * rstd, m = LAYER ? s[LAYER ? 2 : 0] * inv_h : 0.f;
        T* dx = (T*)a.out + j * H;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * NT;
            float gf[VN], o[VN];
            unpack<T>(gv[i], gf);
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                const float n = xf[i][e] * rstd;
                o[e] = rstd * (fmaf(df[i][e], gf[e], -m) - n * c);
                sg[i][e] = fmaf(df[i][e], n, sg[i][e]);
                if (LAYER) sb[i][e] += df[i][e];
            }
            if (v < vpr) Vec<T>::store(dx + v * VN, o);
        }
        if (NT > 64 && !LAYER) __syncthreads();
    };
    for (int64_t j = first; j < n_rows; j += AHEAD * step) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (j + k * step < n_rows) take(x[k], dy[k], j + k * step);
    }
    if (a.pg == nullptr) return;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * NT;
            if (v >= vpr) continue;
#pragma unroll
            for (int q = 0; q < VN / 4; ++q) {
                const int64_t at = (int64_t)blockIdx.x * H + v * VN + 4 * q;
                *reinterpret_cast<float4*>(a.pg + at) = make_float4(sg[i][4 * q], sg[i][4 * q + 1], sg[i][4 * q + 2], sg[i][4 * q + 3]);
                if constexpr (LAYER) {
                    if (a.pb != nullptr)
                        *reinterpret_cast<float4*>(a.pb + at) = make_float4(sb[i][4 * q], sb[i][4 * q + 1], sb[i][4 * q + 2], sb[i][4 * q + 3]);
                }
            }
        }
    } else {
        // the block's four waves, in order
        __shared__ __align__(16) float part[RPB][NV * 64 * VN];
        auto leave = [&](const auto& s, float* out) __attribute__((always_inline)) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int q = 0; q < VN / 4; ++q)
                    *reinterpret_cast<float4*>(&part[threadIdx.x / NT][(tid + i * NT) * VN + 4 * q]) =
                        make_float4(s[i][4 * q], s[i][4 * q + 1], s[i][4 * q + 2], s[i][4 * q + 3]);
            __syncthreads();
            for (int c = threadIdx.x * 4; c < H; c += BT * 4) {
                float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int r = 0; r < RPB; ++r) {
                    const float4 w = *reinterpret_cast<const float4*>(&part[r][c]);
                    t.x += w.x; t.y += w.y; t.z += w.z; t.w += w.w;
                }
                *reinterpret_cast<float4*>(out + (int64_t)blockIdx.x * H + c) = t;
            }
        };
        leave(sg, a.pg);
        if constexpr (LAYER) {
            if (a.pb != nullptr) leave(sb, a.pb);
        }
    }
}

// dg = sum of the blocks' parts (grid.y 1: db): 32 columns a block of 256 threads, 32 groups of parts, in a fixed order
template <typename T, bool MAIN>
__global__ __launch_bounds__(256) void norm_gains_kernel(const float* pg, const float* pb, int n_max, const int32_t* n_dev, int rpb, int blocks, int H,
                                                         void* dg, void* db) {
    __shared__ float red[32][33];
    const int used = norm_bwd_used(live_rows(n_max, n_dev), rpb, blocks);
    const float* p = blockIdx.y == 0 ? pg : pb;
    T* out = (T*)(blockIdx.y == 0 ? dg : db);
    const int cq = threadIdx.x & 7, rg = threadIdx.x >> 3, c0 = blockIdx.x * 32, c = c0 + cq * 4;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < H) {
#pragma unroll 8
        for (int b = rg; b < used; b += 32) {
            const float4 v = *reinterpret_cast<const float4*>(p + (int64_t)b * H + c);
            s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) red[rg][cq * 4 + e] = s[e];
    __syncthreads();
    if (threadIdx.x < 32 && c0 + (int)threadIdx.x < H) {
        float t = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) t += red[r][threadIdx.x];
        if (MAIN) ((float*)out)[c0 + threadIdx.x] += t;
        else out[c0 + threadIdx.x] = narrow_one<T>(t);
    }
}

// Threads a row (a function of the width and the type, so that sums have one order): a wave up to four vectors a lane, which needs no barrier; then the smallest block whose threads hold a row in four.
struct NormShape {
    int nt, rpb;
    NormShape(int dtype, int H) {
        const int vpr = H / (dtype == CF_F32 ? 4 : 8);
        nt = vpr <= 256 ? 64 : vpr <= 1024 ? 256 : 1024;
        rpb = nt == 64 ? 4 : 1;
    }
};
// Blocks of the backward, and so the parts of a gain's gradient: 512, 768 and 1024 take 19.5, 19.8 and 22.2 us (4593 fp32 rows of 840, layer norm: 12.9, 13.4, 15.2)
constexpr int NORM_BWD_BLOCKS = 512;

template <typename T, bool LAYER, bool BWD> static void launch_norm(const RowNormArgs& a, hipStream_t st) {
    const NormShape s(Vec<T>::N == 4 ? CF_F32 : CF_BF16, a.H);
    const int vpr = a.H / Vec<T>::N, nv = (vpr + s.nt - 1) / s.nt;
    const int need = ceil_div(a.n_max, s.rpb), most = BWD ? a.blocks : compute_units() * (s.nt == 1024 ? 2 : 8);
    const int grid = need < most ? need : most;
#define CF_NORM(NT, NV)                                                                                      \
    do {                                                                                                     \
        if constexpr (BWD) norm_bwd_kernel<T, NT, NV, LAYER><<<grid, NT < 256 ? 256 : NT, 0, st>>>(a);       \
        else norm_fwd_kernel<T, NT, NV, LAYER><<<grid, NT < 256 ? 256 : NT, 0, st>>>(a);                     \
    } while (0)
    if (s.nt == 64) {
        if (nv <= 1) CF_NORM(64, 1);
        else if (nv <= 2) CF_NORM(64, 2);
        else CF_NORM(64, 4);
    } else if (s.nt == 256) {
        if (nv <= 2) CF_NORM(256, 2);
        else CF_NORM(256, 4);
    } else {
        if (nv <= 2) CF_NORM(1024, 2);
        else CF_NORM(1024, 4);
    }
#undef CF_NORM
}

template <bool BWD> static void launch_norm_any(const cf_norm_desc& d, const RowNormArgs& a, hipStream_t st) {
    if (d.dtype == CF_F32) d.layer ? launch_norm<float, true, BWD>(a, st) : launch_norm<float, false, BWD>(a, st);
    else d.layer ? launch_norm<bf16_t, true, BWD>(a, st) : launch_norm<bf16_t, false, BWD>(a, st);
}

}  // namespace cf

using namespace cf;

static cf_status norm_check(const cf_norm_desc* d, int32_t max_kept) {
    if (!d) return CF_ERR_NULL;
    if (d->dtype != CF_BF16 && d->dtype != CF_F32) return CF_ERR_DTYPE;
    const int vn = d->dtype == CF_F32 ? 4 : 8;
    if (d->H <= 0 || d->H % vn != 0 || max_kept < 0 || max_kept > (1 << 30) || (d->layer != 0 && d->layer != 1)) return CF_ERR_SHAPE;
    if (!(d->eps >= 0.f) || !(d->eps - d->eps == 0.f)) return CF_ERR_SHAPE;
    return d->H > 4096 * vn ? CF_ERR_UNSUPPORTED : CF_OK;       // a row stays in the registers of a block
}

extern "C" {

cf_status cf_norm_fwd(const cf_norm_desc* desc, const void* x, const void* g, const void* b, const int32_t* idx, const int32_t* n_kept_dev,
                      int32_t max_kept, void* y, cf_stream stream) {
    if (!desc || !x || !g || !y) return CF_ERR_NULL;
    const cf_status ok = norm_check(desc, max_kept);
    if (ok != CF_OK) return ok;
    if (b && !desc->layer) return CF_ERR_SHAPE;
    if (off_by(x, 16) || off_by(g, 16) || off_by(b, 16) || off_by(y, 16) || off_by(idx, 4) || off_by(n_kept_dev, 4)) return CF_ERR_SHAPE;
    const uint64_t bytes = (uint64_t)max_kept * desc->H * dtype_size(desc->dtype);
    const uint64_t row = (uint64_t)desc->H * dtype_size(desc->dtype), known = idx ? row : bytes;          // of x: an index may name few rows
    if (x == y ? idx != nullptr : ranges_meet(x, known, y, bytes)) return CF_ERR_SHAPE;
    if (ranges_meet(y, bytes, g, row) || ranges_meet(y, bytes, b, row)) return CF_ERR_SHAPE;
    if (max_kept == 0) return CF_OK;
    RowNormArgs a{x, g, b, nullptr, idx, n_kept_dev, max_kept, desc->H, desc->eps, y, nullptr, nullptr, 0};
    launch_norm_any<false>(*desc, a, reinterpret_cast<hipStream_t>(stream));
    return hipGetLastError() == hipSuccess ? CF_OK : CF_ERR_HIP;
}

size_t cf_norm_bwd_workspace_bytes(const cf_norm_desc* desc, int32_t max_kept) {
    if (norm_check(desc, max_kept) != CF_OK) return 0;
    const int used = norm_bwd_used(max_kept > 0 ? max_kept : 1, NormShape(desc->dtype, desc->H).rpb, NORM_BWD_BLOCKS);
    return align_up((size_t)(desc->layer ? 2 : 1) * used * desc->H * sizeof(float), 256);
}

cf_status cf_norm_bwd(const cf_norm_desc* desc, const void* x, const void* g, const void* dy_kept, const int32_t* idx, const int32_t* n_kept_dev,
                      int32_t max_kept, void* dx_kept, void* dg, void* db, int32_t main_grad, void* ws, size_t ws_bytes, cf_stream stream) {
    if (!desc || !x || !g || !dy_kept || !dx_kept) return CF_ERR_NULL;
    const cf_status ok = norm_check(desc, max_kept);
    if (ok != CF_OK) return ok;
    if ((db && (!desc->layer || !dg)) || (main_grad != 0 && main_grad != 1)) return CF_ERR_SHAPE;
    for (const void* p : {x, g, dy_kept, (const void*)dx_kept, (const void*)dg, (const void*)db})
        if (off_by(p, 16)) return CF_ERR_SHAPE;
    if (off_by(idx, 4) || off_by(n_kept_dev, 4)) return CF_ERR_SHAPE;
    const uint64_t bytes = (uint64_t)max_kept * desc->H * dtype_size(desc->dtype);
    if (dx_kept != dy_kept && ranges_meet(dx_kept, bytes, dy_kept, bytes)) return CF_ERR_SHAPE;
    const uint64_t row = (uint64_t)desc->H * dtype_size(desc->dtype), known = max_kept == 0 ? 0 : idx ? row : bytes;
    if (dx_kept == x ? idx != nullptr : ranges_meet(dx_kept, bytes, x, known)) return CF_ERR_SHAPE;
    if (ranges_meet(dx_kept, bytes, g, row)) return CF_ERR_SHAPE;
    const uint64_t gb = (uint64_t)desc->H * (main_grad ? 4 : dtype_size(desc->dtype));
    if (ranges_meet(dg, gb, db, gb) || ranges_meet(dg, gb, dx_kept, bytes) || ranges_meet(db, gb, dx_kept, bytes)) return CF_ERR_SHAPE;
    if (dg && (!ws || off_by(ws, 256) || ws_bytes < cf_norm_bwd_workspace_bytes(desc, max_kept))) return CF_ERR_WORKSPACE;
    for (const void* p : {(const void*)dg, (const void*)db})
        if (ranges_meet(p, gb, g, row) || ranges_meet(p, gb, dy_kept, bytes) || ranges_meet(p, gb, x, known)) return CF_ERR_SHAPE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const int rpb = NormShape(desc->dtype, desc->H).rpb;
    const int used = norm_bwd_used(max_kept > 0 ? max_kept : 1, rpb, NORM_BWD_BLOCKS);
    float* pg = dg ? (float*)ws : nullptr;
    float* pb = db ? pg + (size_t)used * desc->H : nullptr;
    RowNormArgs a{x, g, nullptr, dy_kept, idx, n_kept_dev, max_kept, desc->H, desc->eps, dx_kept, pg, pb, NORM_BWD_BLOCKS};
    if (max_kept > 0) launch_norm_any<true>(*desc, a, st);
    if (dg) {
        const dim3 grid(ceil_div(desc->H, 32), db ? 2 : 1);
        if (main_grad) norm_gains_kernel<float, true><<<grid, 256, 0, st>>>(pg, pb, max_kept, n_kept_dev, rpb, NORM_BWD_BLOCKS, desc->H, dg, db);
        else if (desc->dtype == CF_F32) norm_gains_kernel<float, false><<<grid, 256, 0, st>>>(pg, pb, max_kept, n_kept_dev, rpb, NORM_BWD_BLOCKS, desc->H, dg, db);
        else norm_gains_kernel<bf16_t, false><<<grid, 256, 0, st>>>(pg, pb, max_kept, n_kept_dev, rpb, NORM_BWD_BLOCKS, desc->H, dg, db);
    }
    return hipGetLastError() == hipSuccess ? CF_OK : CF_ERR_HIP;
}

}  // extern "C"
