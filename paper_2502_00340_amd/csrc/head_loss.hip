// Loss of kept tokens straight from the head's input x [n, H] and the table E [V, H], with the gradients towards both: the logits s * x E^T are made tile by
// tile in the matrix cores' accumulators and are used up there (but for few fp32 tiles, whose accumulators leave in parts).  What leaves is bounded by the caller's
// workspace:
//
//   1. head_rows      the target's logit of every row, a dot product: ref = s*log2(e) * x.E_y
//   2. head_logits    tiles of x E^T; with t = s*log2(e)*l - ref, strips of 64 columns leave sum(2^t) of the columns that are not the target, and, for the first columns
//                     (as many as the workspace has room for), e = 2^t in the storage type
//   3. head_finish    per row, with q the sum of its strips, lp = -log(1 + q), the loss and its slope; a = -w/norm * dL/dlp * s * exp(lp) is the row's factor: the gradient
//                     of logit c is a * e_c, and a * e'_y with e'_y = expm1(lp) / exp(lp) = -q at the target.  x' = a * x for the table's gradient
//   4. for each piece of the columns (the first one is there already, the others are made again by head_logits):
//      head_dx        slots (+)= e E, fp32          head_dtable   dE (+)= e^T x'
//   5. head_dx_sum    dx = a * sum of the slots
//
// Taking the target's logit as the reference (not the row's maximum, which is not known ahead of the product) makes e a number that needs no second scaling:
// 2^t is at most exp(-lp), so that nothing leaves fp32's or bf16's range unless the target has a probability below exp(-40).  A strip whose sum says so raises its
// row tile's flag; head_logits then goes over the flagged tiles again with strips' maxima, and the row's log-sum-exp becomes its reference.
// The target's own exponential, 1, stays out of the sums: step 1's order of sums is not that of the products, so that 2^t at the target would be 1 + d with a d of some 1e-6, and
// what an almost certain target leaves to the others, 1 - p, would drown in it.  So it keeps all digits, and a row's gradients add up to 0 but for their roundings.
//
// What bounds it: the matrix cores under the chip's power limit from some hundred rows on (4096 rows, H = 4096, V = 128256 bf16: logits, dx and the table's gradient
// 3.07, 3.08 and 3.13 ms, 1.38 to 1.40 PFLOP/s, medians of 12 passes in a row), the table's traffic for few rows.  Keeping e makes that three products instead of four.
//
// Roundings: logits, sums, lp and both gradients' sums are fp32; e, and x' = a*x, are rounded to the storage type once each (2^-8 relative in bf16), dx and
// the table's gradient once where they are stored.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "gemm_tiles.h"
#include "loss_row.h"
#include "mfma_util.h"

namespace cf {

constexpr int STRIP = 64;                       // columns that share a sum
constexpr float FLAG_ABOVE = 288230376151711744.f;      // 2^58 = exp(40): a strip's sum beyond it asks for another reference

struct HeadArgs {
    const void *x, *table;
    int H, V, n_max;
    const int32_t* n_dev;
    float k;                // logit scale * log2(e)
    int ldn, strips;        // rows of the strips' array; sums that a row has where its tile is not flagged
    float *ref, *sums;      // [n_max]; [strips][ldn]
    float *a, *ey;          // [n_max]: the row's factor; e at the target
    int32_t *y, *flags;     // target or -1; flags[0]: any, flags[1 + i]: rows 256 i ..
    void* e;                // [n_max, lde]: columns c0 .. c0 + lde - 1
    int lde, c0, c1;        // the launch's columns: c0 .. c1 - 1
    int store_end;          // columns below it are stored
    bool flagged_only;
    float* part;            // fp32: [parts] tiles' accumulators of each part of the contraction, where it is cut
    int parts;
};
enum HeadKind { SUMS = 0, MAXIMA = 1, VALUES = 2 };

// ---- 1. targets --------------------------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(256) void head_rows_kernel(HeadArgs a, LossArgs l) {
    constexpr int VN = Vec<T>::N;
    const int n_rows = live_rows(a.n_max, a.n_dev), lane = threadIdx.x & 63;
    const int n_flags = (a.n_max + 255) / 256 + 1;
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < n_flags; i += 256) a.flags[i] = 0;
    for (int64_t j = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); j < n_rows; j += (int64_t)gridDim.x * 4) {
        const int64_t row = l.idx != nullptr ? l.idx[j] : j, t = l.targets[row];
        const bool live = t >= 0 && t < a.V && (l.weights == nullptr || l.weights[row] != 0.f);
        float s = 0.f;
        if (live) {
            const T *x = (const T*)a.x + j * a.H, *w = (const T*)a.table + t * a.H;
            for (int c = lane * VN; c < a.H; c += 64 * VN) {
                float p[VN], q[VN];
                Vec<T>::load(x + c, p);
                Vec<T>::load(w + c, q);
#pragma unroll
                for (int e = 0; e < VN; ++e) s = fmaf(p[e], q[e], s);
            }
        }
        s = wave_sum(s);
        if (lane == 0) {
            // +inf stands for a row that is left out: its 2^t is 0 whatever t; a live row whose logit is +inf has no finite probability at all
            const float r = s * a.k;
            a.ref[j] = live ? (r == INFINITY ? NAN : r) : INFINITY;
            a.ey[j] = fmaf(s, a.k, -r);         // what rounding left, for head_finish
            a.y[j] = live ? (int32_t)t : -1;
        }
    }
}

// ---- 2. tiles of logits ------------------------------------------------------------------------------------

template <int KIND> struct LeaveLogits {
    static constexpr bool OWN = true, LDA = false, STREAM = false;
    HeadArgs a;
    int n_rows;
    struct Rows {
        float ref[8], ey[KIND == VALUES ? 8 : 1];
        int y[8];
    };
    template <int TM> __device__ __forceinline__ Rows rows(const TileRef& t, int wm) const {
        Rows r;
#pragma unroll
        for (int i = 0; i < 2 * TM; ++i) {
            const int m = t.m0 + wm * (32 * TM) + i * 16 + (threadIdx.x & 15), at = min(m, n_rows - 1);
            const float ref = a.ref[at];
            const int y = a.y[at];
            r.ref[i] = m < n_rows ? ref : INFINITY;
            r.y[i] = m < n_rows ? y : -1;
            if constexpr (KIND == VALUES) r.ey[i] = a.ey[at];
        }
        // arrived ahead of whatever is asked for next
#pragma unroll
        for (int i = 0; i < 2 * TM; ++i) {
            asm volatile("" : "+v"(r.ref[i]));
            asm volatile("" : "+v"(r.y[i]));
            if constexpr (KIND == VALUES) asm volatile("" : "+v"(r.ey[i]));
        }
        return r;
    }
    template <int TM, int TN>
    __device__ __forceinline__ void operator()(f32x4_t (&acc)[2 * TM][2 * TN], const TileRef& t, const Rows& row, unsigned char* smem, int wm, int wn) const {
        // Columns behind the last one, in the last column of tiles, and targets among a wave's rows and columns have a copy of the code of their own: a write to the
        // accumulators, or a branch around a part of this, would have all of them copied to vector registers, and others spilled
        bool hit = false;
#pragma unroll
        for (int i = 0; i < 2 * TM; ++i) hit |= (unsigned)(row.y[i] - (t.n0 + wn * (32 * TN))) < 32u * TN;
        if (t.n0 + 64 * TN > a.V) write_out<TM, TN, true, true>(acc, t, row, smem, wm, wn);
        else if (__any(hit)) write_out<TM, TN, false, true>(acc, t, row, smem, wm, wn);
        else write_out<TM, TN, false, false>(acc, t, row, smem, wm, wn);
    }
    template <int TM, int TN, bool EDGE, bool TARGETS>
    __device__ __forceinline__ void write_out(f32x4_t (&acc)[2 * TM][2 * TN], const TileRef& t, const Rows& row, unsigned char* smem, int wm, int wn) const {
        constexpr int FN = 2 * TN, NS = FN / 4;
        const int rows = n_rows;
        int ln = threadIdx.x & 63;
        asm volatile("" : "+v"(ln));            // rebuilt for each tile, not carried through the products
        const int l16 = ln & 15, g4 = ln >> 4;
        const int n0 = t.n0 + wn * (32 * TN), mw = t.m0 + wm * (32 * TM), left = a.V - n0 - 4 * g4;
        const bool store = KIND != MAXIMA && t.n0 < a.store_end;
        constexpr int RBY = 64 * TN, CPR = RBY / 16, RPP = 64 / CPR, NP = 32 / RPP, NV = CPR / RPP;     // as in the products' own write-out
        unsigned char* stg = smem + GEMM_RING + ((wm * 2 + wn) * 8192);
        const int c = ln % CPR, rl = ln / CPR, col = n0 + c * 8;
        const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(
            (bf16_t*)a.e + (int64_t)mw * a.lde, 0, store ? max(0, min(rows - mw, 32 * TM)) * a.lde * 2 : 0, 0x00020000);       // nothing is stored: an empty range
        const unsigned voff = col - a.c0 < a.lde ? (unsigned)(rl * a.lde + (col - a.c0)) * 2u : 0x80000000u;
        const unsigned char* rd[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) rd[v] = stg + rl * RBY + ((c ^ ((rl + RPP * v) & (CPR - 1))) << 4);
        unsigned char* const wr = stg + l16 * RBY + (g4 & 1) * 8;
        const int wsw = l16 & (CPR - 1), wch = g4 >> 1;
        float* const sums = a.sums + (int64_t)(n0 / STRIP) * a.ldn + mw + l16;
        bool beyond = false;
#pragma unroll
        for (int i2 = 0; i2 < TM; ++i2) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = 2 * i2 + h;
                const float ref = row.ref[i];
                const bool dead = ref == INFINITY;
                const int yrel = row.y[i] - n0 - 4 * g4;
                const float ey = row.ey[KIND == VALUES ? i : 0];
                const unsigned mask = dead ? 0u : ~0u;          // whatever such a row holds, NaN included
#pragma unroll
                for (int z = 0; z < NS; ++z) {
                    float s = 0.f, mx = -INFINITY;
                    if constexpr (KIND == MAXIMA) {
#pragma unroll
                        for (int j = 4 * z; j < 4 * z + 4; ++j)
#pragma unroll
                            for (int v = 0; v < 4; ++v) mx = (!EDGE || j * 16 + v < left) && (!TARGETS || j * 16 + v != yrel) ? fmaxf(mx, acc[i][j][v]) : mx;
                        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                        mx *= a.k;
                    }
                    const float r = KIND == MAXIMA ? (mx == -INFINITY ? 0.f : mx) : ref;
#pragma unroll
                    for (int j = 4 * z; j < 4 * z + 4; ++j) {
                        float e[4];
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            e[v] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][v], a.k, -r));
                            if constexpr (EDGE) e[v] = j * 16 + v < left ? e[v] : 0.f;
                            if constexpr (TARGETS) e[v] = yrel == j * 16 + v ? (KIND == VALUES ? ey : 0.f) : e[v];
                            if constexpr (KIND != VALUES) s += e[v];
                        }
                        if constexpr (KIND != MAXIMA) {
                            uint2 o;
                            o.x = pack_bf16x2(e[0], e[1]) & mask;
                            o.y = pack_bf16x2(e[2], e[3]) & mask;
                            *reinterpret_cast<uint2*>(wr + h * 16 * RBY + (((2 * j + wch) ^ wsw) << 4)) = o;
                        }
                    }
                    if constexpr (KIND != VALUES) {
                        s += __shfl_xor(s, 16, 64);
                        s += __shfl_xor(s, 32, 64);
                        if (KIND == SUMS) beyond |= !dead && !(s <= FLAG_ABOVE);
                        if (g4 == 0 && mw + i * 16 + l16 < rows && (!EDGE || n0 + z * STRIP < a.V)) sums[(int64_t)z * a.ldn + i * 16] = KIND == MAXIMA ? mx + log2f(s) : s;
                    }
                    CF_SCHED_FENCE();       // strip by strip: what is spilled comes back behind the next tile's loads
                }
            }
            if constexpr (KIND != MAXIMA) {
                u32x4_t val[NP];
#pragma unroll
                for (int q = 0; q < NP; ++q) val[q] = *reinterpret_cast<const u32x4_t*>(rd[q % NV] + q * RPP * RBY);
#pragma unroll
                for (int q = 0; q < NP; ++q)
                    __builtin_amdgcn_raw_buffer_store_b128(val[q], rc, voff + (unsigned)((i2 * 32 + q * RPP) * a.lde) * 2u, 0, 0);
                CF_SCHED_FENCE();
            }
        }
        if (KIND == SUMS && beyond) a.flags[0] = a.flags[1 + (t.m0 >> 8)] = 1;
    }
};

// The tiles of x E^T over the launch's columns, as a product's: whole 256x256 ones that fill rounds of the CUs, then the rest in smaller ones.
template <int KIND> __global__ __launch_bounds__(256) void head_logits_kernel(HeadArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    if (a.flagged_only && __builtin_amdgcn_readfirstlane(a.flags[0]) == 0) return;
    const int rows = __builtin_amdgcn_readfirstlane(live_rows(a.n_max, a.n_dev)), width = a.c1 - a.c0;
    const int tiles_m = (rows + 255) / 256, tiles_n = (width + 255) / 256, tiles = tiles_m * tiles_n;
    int n_full, sub;
    plan_tiles(tiles, (int)gridDim.x, n_full, sub);
    if (rows <= 128) { n_full = 0; sub = 4; }           // half of a whole tile's rows would not exist
    n_full = __builtin_amdgcn_readfirstlane(n_full);
    sub = __builtin_amdgcn_readfirstlane(sub);
    const int n_items = n_full + (tiles - n_full) * sub, stride = (int)gridDim.x;
    GemmArgs g;
    g.A[0] = a.x; g.B[0] = a.table; g.K[0] = a.H; g.nseg = 1; g.C = nullptr; g.M = rows; g.N = a.c1; g.alpha = 1.f; g.beta = 0.f;
    g.a_idx = nullptr; g.a_rows = 0; g.n_dev = nullptr; g.lda = a.H;
    auto decode = [&](int w, TileRef& t) __attribute__((always_inline)) {
        int bm, bn, m0, n0;
        if (w < n_full) {
            tile_coords(xcd_order(w, n_full), tiles_m, tiles_n, bm, bn);
            m0 = bm * 256;
            n0 = bn * 256;
        } else {
            const int j = xcd_order(w - n_full, n_items - n_full), part = j % sub;
            tile_coords(n_full + j / sub, tiles_m, tiles_n, bm, bn);
            m0 = bm * 256 + (sub == 4 ? (part >> 1) * 128 : 0);
            n0 = bn * 256 + (sub == 4 ? (part & 1) * 128 : (sub == 2 ? part * 128 : 0));
            if (m0 >= rows || n0 >= width) return false;
        }
        if (a.flagged_only && __builtin_amdgcn_readfirstlane(a.flags[1 + bm]) == 0) return false;
        n0 += a.c0;
        t.m0 = __builtin_amdgcn_readfirstlane(m0);
        t.n0 = __builtin_amdgcn_readfirstlane(n0);
        t.M = rows;
        t.N = __builtin_amdgcn_readfirstlane(min(a.c1, n0 + 256));      // the descriptor of a tile's rows of the table spans these rows alone
        t.A0 = uniform_ptr(a.x);
        t.B0 = uniform_ptr(a.table);
        t.C = nullptr;
        return true;
    };
    const LeaveLogits<KIND> leave{a, rows};
    int w = (int)blockIdx.x;
    TileRef t;
    auto seek = [&](int end) __attribute__((always_inline)) {       // this block's first live item from w on
        for (; w < end; w += stride)
            if (decode(w, t)) return true;
        return false;
    };
    auto next_in = [&](int end) {
        return [&, end](TileRef& nx) __attribute__((always_inline)) {
            w += stride;
            if (!seek(end)) return false;
            nx = t;
            return true;
        };
    };
    if (seek(n_full)) gemm_tiles<0, 4, 4, false, false>(g, a.H, t, next_in(n_full), smem, 0, 0, nullptr, leave);
    if (!seek(n_items)) return;
    if (sub == 1) gemm_tiles<0, 4, 4, false, false>(g, a.H, t, next_in(n_items), smem, 0, 0, nullptr, leave);
    else if (sub == 2) gemm_tiles<0, 4, 2, false, false>(g, a.H, t, next_in(n_items), smem, 0, 0, nullptr, leave);
    else gemm_tiles<0, 2, 2, false, false>(g, a.H, t, next_in(n_items), smem, 0, 0, nullptr, leave);
}

// Few rows: the table's traffic counts, not the products.  A block of eight waves walks through tiles of 128 rows of the table, which go from memory
// straight into the registers that the MFMAs take them from, P steps of 64 k ahead; x, 16 * NF rows of 64 k a step, lies in a ring in LDS that all waves
// fill and read.  Each wave keeps the sums of its columns over all its tiles: one value a row and block leaves.  The loads never stop, between tiles neither.
// Blocks begin a row's k at different places: rows of the table are a power of two apart as a rule, and blocks that all read the same part of theirs meet in
// the same memory channels (64 rows of x, [128256, 4096]: 217 us, and 176 so, 6.0 TB/s; tiles of 256 rows 241 and 180; 128x128 product tiles 289).
template <int NF, int P> __global__ __launch_bounds__(512) void head_few_kernel(HeadArgs a) {
    constexpr int R = P + 1, ROWS = 16 * NF, SLOT = ROWS * 128, XL = NF > 4 ? NF / 4 : 1, NB = 2;            // XL, NB: loads of a wave and step
    extern __shared__ __align__(16) unsigned char smem[];
    unsigned char* const stage = smem + R * SLOT;       // a tile's exponentials, [row][128 columns], 16-byte chunks XOR-ed with the row
    __shared__ float red[8][ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int rows = __builtin_amdgcn_readfirstlane(live_rows(a.n_max, a.n_dev)), H = a.H, steps = (H + 63) / 64;
    if (rows == 0) return;
    constexpr int TILE = 128;
    const int tiles = (a.V + TILE - 1) / TILE;
    const i32x4_t rx = make_rsrc(a.x, (int64_t)rows * H * 2);
    constexpr unsigned OOB = 0x80000000u;
    unsigned xoff[XL];
    int xk[XL];
    unsigned xdst[XL];
#pragma unroll
    for (int u = 0; u < XL; ++u) {
        const int part = (wave + 8 * u) % (2 * NF), row = part * 8 + (lane >> 3);       // of the slot; with few rows several waves load the same part
        xk[u] = ((lane & 7) ^ nt_swz(row)) * 8;
        xoff[u] = (unsigned)row * (unsigned)H * 2u + xk[u] * 2u;
        xdst[u] = __builtin_amdgcn_readfirstlane(lds_addr_of(smem) + part * 1024);
    }
    // (tile, step) that the next loads fetch
    const int rot = (int)(blockIdx.x * 37u) % steps;
    int lt = blockIdx.x, ls = 0, slot_in = 0;
    __amdgpu_buffer_rsrc_t rb;
    auto open = [&]() __attribute__((always_inline)) {
        const int64_t v0 = (int64_t)lt * TILE;
        const int64_t have = lt < tiles ? min((int64_t)TILE, a.V - v0) : 0;
        rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>((const bf16_t*)a.table + (lt < tiles ? v0 : 0) * H), 0, (int)(have * H * 2), 0x00020000);
    };
    open();
    const unsigned boff = (unsigned)(wave * 16 + l16) * (unsigned)H * 2u + g4 * 16u;
    u32x4_t b[P][NB];
    auto fetch = [&](u32x4_t (&to)[NB]) __attribute__((always_inline)) {
        const int k0 = (ls + rot >= steps ? ls + rot - steps : ls + rot) * 64;
#pragma unroll
        for (int u = 0; u < XL; ++u)
            dma16s(xdst[u] + slot_in * SLOT, rx, k0 + xk[u] < H ? xoff[u] : OOB, (unsigned)k0 * 2u);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            to[ks] = __builtin_amdgcn_raw_buffer_load_b128(rb, k0 + ks * 32 + g4 * 8 < H ? boff : OOB, (k0 + ks * 32) * 2, 0);
        CF_SCHED_FENCE();
        slot_in = slot_in + 1 == R ? 0 : slot_in + 1;
        if (++ls == steps) {
            ls = 0;
            lt += (int)gridDim.x;
            open();
        }
    };
    float ref[NF], sum[NF];
    int y[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        const int m = i * 16 + l16;
        ref[i] = m < rows ? a.ref[m] : INFINITY;
        y[i] = m < rows ? a.y[m] : -1;
        sum[i] = 0.f;
    }
#pragma unroll
    for (int p = 0; p < P; ++p) fetch(b[p]);
    f32x4_t acc[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    int tile = blockIdx.x, s = 0, slot = 0;
    auto leave = [&]() __attribute__((always_inline)) {
        const int c = tile * TILE + wave * 16 + 4 * g4;
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            float e[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                e[v] = __builtin_amdgcn_exp2f(fmaf(acc[i][v], a.k, -ref[i]));
                e[v] = c + v < a.V && c + v != y[i] ? e[v] : 0.f;
                sum[i] += e[v];
            }
            if (a.store_end > 0) {
                const bool dead = ref[i] == INFINITY;
                uint2 o;
                o.x = dead ? 0u : pack_bf16x2(e[0], e[1]);
                o.y = dead ? 0u : pack_bf16x2(e[2], e[3]);
                *reinterpret_cast<uint2*>(stage + (i * 16 + l16) * 256 + (((2 * wave + (g4 >> 1)) ^ l16) << 4) + (g4 & 1) * 8) = o;
            }
        }
        if (a.store_end == 0 || tile * TILE >= a.lde) return;
        lds_barrier();          // the next one that writes here has the barrier of a step ahead of it
        for (int v = threadIdx.x; v < rows * 16; v += 512) {            // whole rows of the tile; zeros behind the last column, too
            const int m = v >> 4, ch = v & 15, col = tile * TILE + ch * 8;
            if (col < a.lde)
                *reinterpret_cast<u32x4_t*>((bf16_t*)a.e + (int64_t)m * a.lde + col) = *reinterpret_cast<const u32x4_t*>(stage + m * 256 + ((ch ^ (m & 15)) << 4));
        }
    };
    const int frag = l16 * 128, ch0 = (g4 ^ nt_swz(l16)) << 4, ch1 = ((4 + g4) ^ nt_swz(l16)) << 4;
    // Whole rounds of P steps (the steps behind the last tile's run on zeros, and nothing takes what they give): a way out in the middle would have the compiler wait for
    // the youngest load at the loop's head
    const int mine = (tiles - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
    for (int64_t left = (int64_t)mine * steps; left > 0; left -= P) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            wait_vmcnt<(P - 1) * (XL + NB)>();
            lds_barrier();              // the step's rows of x are there, and every wave is done with the step before
            const unsigned char* xs = smem + slot * SLOT + frag;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < NF; ++i) {
                    const bf16x8_t fa = *reinterpret_cast<const bf16x8_t*>(xs + i * 2048 + (ks ? ch1 : ch0));
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, b[p][ks]), fa, acc[i], 0, 0, 0);
                }
            CF_SCHED_FENCE();
            fetch(b[p]);
            slot = slot + 1 == R ? 0 : slot + 1;
            if (++s == steps) {
                if (tile < tiles) leave();
#pragma unroll
                for (int i = 0; i < NF; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                s = 0;
                tile += (int)gridDim.x;
            }
        }
    }
    wait_vmcnt<0>();            // loads into LDS must not outlive the block
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        sum[i] += __shfl_xor(sum[i], 16, 64);
        sum[i] += __shfl_xor(sum[i], 32, 64);
        if (g4 == 0) red[wave][i * 16 + l16] = sum[i];
    }
    __syncthreads();
    for (int m = threadIdx.x; m < rows; m += 512) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += red[w][m];
        a.sums[(int64_t)blockIdx.x * a.ldn + m] = t;
        if (a.ref[m] != INFINITY && !(t <= FLAG_ABOVE)) a.flags[0] = a.flags[1] = 1;
    }
}

static int few_blocks(int V, int n_cu) { return std::min(ceil_div(V, 128), n_cu); }
constexpr int FEW_ROWS = 128;

// ---- 3. the rows' ends -------------------------------------------------------------------------------------
// A block takes 16 rows: 64 groups of 16 lanes add their strips up, one lane a row ends it, and the block scales the rows of x.  A single block has all terms, and leaves
// the statistics, too.
template <typename T>
__global__ __launch_bounds__(1024) void head_finish_kernel(HeadArgs a, LossArgs l, void* xs, float* stats) {
    constexpr int VN = Vec<T>::N;
    __shared__ float red[2][16][16];
    __shared__ float fac[16], terms[16][4];
    const int n_rows = live_rows(a.n_max, a.n_dev), j0 = blockIdx.x * 16, tid = threadIdx.x, r = tid & 15, grp = tid >> 4, j = j0 + r;
    if (j0 >= n_rows) {
        if (stats != nullptr && tid < 4) stats[tid] = 0.f;
        return;
    }
    const bool flagged = a.flags[1 + (j0 >> 8)] != 0;           // the same for the 16 rows
    const int strips = flagged ? (a.V + STRIP - 1) / STRIP : a.strips;
    float m = 0.f, s = 0.f;
    if (!flagged) {
        if (j < n_rows) {
#pragma unroll 8
            for (int i = grp; i < strips; i += 64) s += a.sums[(int64_t)i * a.ldn + j];
        }
    } else {
        m = -INFINITY;
        if (j < n_rows)
            for (int i = grp; i < strips; i += 64) {            // log2 of each strip's sum
                const float t = a.sums[(int64_t)i * a.ldn + j], n = fmaxf(m, t);
                if (t == -INFINITY) continue;
                s = s * __builtin_amdgcn_exp2f(m - n) + __builtin_amdgcn_exp2f(t - n);
                m = n;
            }
#pragma unroll
        for (int o = 16; o < 64; o <<= 1) {
            const float mo = __shfl_xor(m, o, 64), so = __shfl_xor(s, o, 64), n = fmaxf(m, mo);
            if (n != -INFINITY) s = s * __builtin_amdgcn_exp2f(m - n) + so * __builtin_amdgcn_exp2f(mo - n);
            m = n;
        }
    }
    if (!flagged) {
        s += __shfl_xor(s, 16, 64);
        s += __shfl_xor(s, 32, 64);
    }
    if ((tid & 63) < 16) { red[0][tid >> 6][r] = m; red[1][tid >> 6][r] = s; }
    __syncthreads();
    if (tid < 16 && j < n_rows) {
        m = red[0][0][r];
#pragma unroll
        for (int w = 1; w < 16; ++w) m = fmaxf(m, red[0][w][r]);
        s = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            const float t = red[1][w][r];
            s += !flagged ? t : t == 0.f ? 0.f : t * __builtin_amdgcn_exp2f(red[0][w][r] - m);
        }
        const int y = a.y[j];
        float lp = 0.f, fy = 0.f;
        RowLoss rl{make_float4(0.f, 0.f, 0.f, 0.f), 0.f};
        if (y >= 0) {
            // q: what the other columns' exponentials add up to relative to the target's own, lp = -log(1 + q).  s is relative to ref, the target's logit but for its
            // rounding r, or, flagged, to m
            const float ref = a.ref[j], ln2 = 0.6931471805599453f, r = ln2 * a.ey[j];
            float fy0, ey;          // the row's factor is the slope times fy0
            if (!flagged) {
                const float by = expf(-r), q = s * by;
                lp = -log1pf(q);
                fy0 = by / (1.f + q);
                ey = -s;
            } else {
                const float t = ln2 * (m - ref) + (logf(s) - r), small = log1pf(expf(-fabsf(t))), log2e = 1.4426950408889634f;         // t = log(q)
                lp = -(fmaxf(t, 0.f) + small);
                const float lse = (t > 0.f ? m + log2f(s) : ref) + small * log2e;
                a.ref[j] = lse == INFINITY ? NAN : lse;
                fy0 = 1.f;
                ey = expm1f(lp);
            }
            RowHead h;
            h.row = l.idx != nullptr ? l.idx[j] : j;
            h.y = y;
            h.w = l.weights != nullptr ? l.weights[h.row] : 1.f;
            h.old = h.ref = h.adv = 0.f;
            if (l.policy) {
                h.old = l.old_logp[h.row];
                h.adv = l.adv[h.row];
                if (l.ref_logp != nullptr) h.ref = l.ref_logp[h.row];
            }
            rl = row_loss(l, h, lp, 1.f / (l.norm != 0.f ? l.norm : (float)n_rows));
            fy = -rl.coef * l.scale * fy0;
            if constexpr (sizeof(T) == 2) {
                // The target's e is most of a row's gradient.  Its rounding goes over to the row's factor, so that factor times e is exact at the target and
                // off by that rounding, and their own, at the other columns: gradients 1.4 times as far off as one rounding instead of 1.7.
                const float near = bf16_to_f32(narrow_one<bf16_t>(ey)), by = ey / near;
                if (by > 0.5f && by < 2.f) fy *= by;
                ey = near;
            }
            a.ey[j] = ey;
            if (a.e != nullptr && !flagged && y < a.store_end) ((T*)a.e)[(int64_t)j * a.lde + y] = narrow_one<T>(ey);
        }
        a.a[j] = fy;
        fac[r] = fy;
        if (l.logp != nullptr) l.logp[j] = lp;
        l.terms[j] = rl.terms;
        terms[r][0] = rl.terms.x; terms[r][1] = rl.terms.y; terms[r][2] = rl.terms.z; terms[r][3] = rl.terms.w;
    }
    if (xs == nullptr && stats == nullptr) return;
    __syncthreads();
    const int vpr = a.H / VN, rows = min(16, n_rows - j0);
    if (stats != nullptr && tid < 4) {
        double t = 0.;
        for (int i = 0; i < rows; ++i) t += terms[i][tid];
        stats[tid] = (float)(t / (l.norm != 0.f ? (double)l.norm : (double)n_rows));
    }
    if (xs == nullptr) return;
    for (int v = tid; v < rows * vpr; v += 1024) {
        const int q = v / vpr;
        const int64_t at = (int64_t)(j0 + q) * a.H + (v - q * vpr) * VN;
        float o[VN];
        Vec<T>::load((const T*)a.x + at, o);
#pragma unroll
        for (int e = 0; e < VN; ++e) o[e] = a.y[j0 + q] < 0 ? 0.f : o[e] * fac[q];
        Vec<T>::store((T*)xs + at, o);
    }
}

// ---- 4. products of a piece --------------------------------------------------------------------------------

// dx: e [n, K] times the piece's rows of the table [K, H], fp32 tiles that the first piece writes and the others add to.  The tiles that do not fill a round of the
// resident blocks have their contraction cut into parts: the first part lies with the whole tiles in slots [n, H], the others in tiles of their own, for
// head_dx_sum_kernel to add up.  All of it is a function of the live rows: kernels agree on it whoever knows the count.  (4096 rows, [65536, 4160], 272 tiles: all
// of them in parts 2395 us, 1804 so.)
struct DxPlan {
    int tm, tn, n_full, rem, parts;
    __device__ DxPlan(int rows, int H, int V, int tile, int resident) {
        tm = (rows + tile - 1) / tile;
        tn = (H + tile - 1) / tile;
        n_full = tm * tn / resident * resident;
        rem = tm * tn - n_full;
        parts = 1;
        if (rem > 0) {          // one round, or two where these are shorter
            const int one = resident / rem, two = 2 * resident / rem;
            parts = 20 * one < 17 * (two - one) ? two : one;
            parts = max(1, min(min(parts, 64), V / 512));
        }
    }
    __device__ int items() const { return n_full + rem * parts; }
    // item -> tile (in the order of tile_coords) and part
    __device__ void item(int w, int& tile, int& part) const {
        part = 0;
        if (w < n_full) { tile = xcd_order(w, n_full); return; }
        const int l = xcd_order(w - n_full, rem * parts);
        part = l / rem;
        tile = n_full + l - part * rem;
    }
    // where an element (row, col) of a part lies: offset from `more` of parts 1 .. for one of the tiles behind the whole ones
    __device__ int64_t more(int tile, int part, int side) const { return ((int64_t)(tile - n_full) * (parts - 1) + part - 1) * side * side; }
};

struct LeaveSlots {
    static constexpr bool OWN = true, LDA = true, STREAM = false;
    float* origin;              // of the tile
    int ld;
    bool first;
    struct Rows {};
    template <int TM> __device__ __forceinline__ Rows rows(const TileRef&, int) const { return {}; }
    template <int TM, int TN>
    __device__ __forceinline__ void operator()(f32x4_t (&acc)[2 * TM][2 * TN], const TileRef& t, const Rows&, unsigned char*, int wm, int wn) const {
        constexpr int FM = 2 * TM, FN = 2 * TN;
        int ln = threadIdx.x & 63;
        asm volatile("" : "+v"(ln));
        const int mw = t.m0 + wm * (32 * TM), have = min(t.M - mw, 32 * TM), col = wn * (32 * TN) + 4 * (ln >> 4), n = t.n0 + col;
        const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(origin + (int64_t)(wm * (32 * TM)) * ld, 0, have > 0 ? have * ld * 4 : 0, 0x00020000);
        const unsigned row_bytes = (unsigned)ld * 4u, voff = (unsigned)(ln & 15) * row_bytes + (unsigned)col * 4u;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            u32x4_t old[FN];
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                old[j] = u32x4_t{0u, 0u, 0u, 0u};
                if (!first)
                    old[j] = __builtin_amdgcn_raw_buffer_load_b128(rc, n + j * 16 < t.N ? voff + (unsigned)(i * 16) * row_bytes + j * 64u : 0x80000000u, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                u32x4_t o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(acc[i][j][e] + __uint_as_float(old[j][e]));
                __builtin_amdgcn_raw_buffer_store_b128(o, rc, n + j * 16 < t.N ? voff + (unsigned)(i * 16) * row_bytes + j * 64u : 0x80000000u, 0, 0);
            }
            CF_SCHED_FENCE();
        }
    }
};
struct DxArgs {
    const void *e, *table;      // the piece's rows of the table
    int lde, K, H, n_max;
    const int32_t* n_dev;
    float *slots, *more;
    int V, tile, resident;      // tile: 256 or 128
    bool first;
};
__global__ __launch_bounds__(256) void head_dx_kernel(DxArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int rows = __builtin_amdgcn_readfirstlane(live_rows(a.n_max, a.n_dev));
    const DxPlan plan(rows, a.H, a.V, a.tile, a.resident);
    const int items = plan.items(), pairs = (a.K + 63) / 64;
    GemmArgs g;
    g.A[0] = a.e; g.B[0] = a.table; g.K[0] = a.K; g.nseg = 1; g.C = nullptr; g.M = rows; g.N = a.H; g.alpha = 1.f; g.beta = 0.f;
    g.a_idx = nullptr; g.a_rows = 0; g.n_dev = nullptr; g.lda = a.lde;
    auto none = [](TileRef&) { return false; };
    for (int w = blockIdx.x; w < items; w += gridDim.x) {
        int tile, part, bm, bn;
        plan.item(w, tile, part);
        tile = __builtin_amdgcn_readfirstlane(tile);
        part = __builtin_amdgcn_readfirstlane(part);
        tile_coords(tile, plan.tm, plan.tn, bm, bn);
        TileRef t{__builtin_amdgcn_readfirstlane(bm * a.tile), __builtin_amdgcn_readfirstlane(bn * a.tile), rows, a.H, uniform_ptr(a.e),
                  uniform_ptr(a.table), nullptr};
        const LeaveSlots leave{part == 0 ? a.slots + (int64_t)t.m0 * a.H + t.n0 : a.more + plan.more(tile, part, a.tile), part == 0 ? a.H : a.tile, a.first};
        const int per = tile < plan.n_full ? pairs : (pairs + plan.parts - 1) / plan.parts;
        const int pbeg = min(pairs, part * per), pend = min(pairs, pbeg + per);
        if (a.tile == 256) gemm_tiles<2, 4, 4, true, false>(g, a.K, t, none, smem, pbeg, pend, nullptr, leave);
        else gemm_tiles<2, 2, 2, true, false>(g, a.K, t, none, smem, pbeg, pend, nullptr, leave);
        wait_vmcnt<0>();
        lds_barrier();
    }
}

// the table's gradient: e^T x' over the live rows, bf16 written (past the caches: nothing here reads it, and e and x' stay in them; whole calls 0.985 to 0.997 of
// the time) or fp32 added to
struct WideA : Product {
    static constexpr bool LDA = true, STREAM = true;
};
struct DtableArgs {
    const void *e, *xs;
    void* out;                  // the piece's rows of the gradient
    int lde, K, H, n_max;       // K: the piece's rows
    const int32_t* n_dev;
    int n_full, sub;
};
template <bool CF32> __global__ __launch_bounds__(256) void head_dtable_kernel(DtableArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int rows = __builtin_amdgcn_readfirstlane(live_rows(a.n_max, a.n_dev));
    const int tm = (a.K + 255) / 256, tn = (a.H + 255) / 256;
    GemmArgs g;
    g.A[0] = a.e; g.B[0] = a.xs; g.K[0] = rows; g.nseg = 1; g.C = a.out; g.M = a.K; g.N = a.H; g.alpha = 1.f; g.beta = 0.f;
    g.a_idx = nullptr; g.a_rows = 0; g.n_dev = nullptr; g.lda = a.lde;
    gemm_items<1, CF32, WideA>(g, rows, tm * tn, a.n_full, a.sub, (int)gridDim.x, [&](int l, TileRef& t, int& bm, int& bn) __attribute__((always_inline)) {
        t = TileRef{0, 0, a.K, a.H, a.e, a.xs, a.out};
        tile_coords(l, tm, tn, bm, bn);
    }, smem);
}

// The same for few rows, a write of the gradient with little to compute: a block holds the fragments of x' for 256 columns in its registers and walks through
// tiles of 64 rows of the table, whose exponentials it reads transposed from LDS.  A lane's four fragments of x' are columns 16 * (l / 16) + 4 j .. +3 of its wave's 64,
// so that it ends up with 16 adjacent columns of a row of the gradient.
constexpr int DT_FEW_ROWS = 128, DT_TILE = 64;
template <int KS, bool CF32> __global__ __launch_bounds__(256) void head_dtable_few_kernel(DtableArgs a, int per) {
    constexpr int ROWS = 32 * KS;
    __shared__ __align__(16) unsigned char xs[ROWS * 512];          // [row][256 columns], then twice [row][64 columns of e]
    const int rows = live_rows(a.n_max, a.n_dev), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, g4 = lane >> 4;
    const int hb = (a.H + 255) / 256, h0 = (int)blockIdx.x % hb * 256, tiles = (a.K + DT_TILE - 1) / DT_TILE;
    const int first = (int)blockIdx.x / hb * per, end = min(tiles, first + per);
    if (first >= end) return;
    // fragments are read transposed; of a row's chunks of 16 bytes those of 64 are XOR-ed with its number, so that the four rows of a read fall into different banks
    auto swz = [](int k, bool wide) { return wide ? (k & 3) << 2 : (k & 2) << 1; };
    auto frag = [&](unsigned char* s, bool wide, int ks, int col0) __attribute__((always_inline)) {
        const int row_bytes = wide ? 512 : 128, kl = ks * 32 + 8 * g4 + (l16 >> 2), ch = col0 / 8 + ((lane & 3) >> 1);
        unsigned char* p = s + kl * row_bytes + ((ch ^ swz(kl, wide)) << 4) + (lane & 1) * 8;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(__attribute__((address_space(3))) unsigned char*)p);
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(__attribute__((address_space(3))) unsigned char*)(p + 4 * row_bytes));
        return __builtin_bit_cast(bf16x8_t, (s16x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const u32x4_t zero = {0u, 0u, 0u, 0u};
    for (int v = tid; v < ROWS * 32; v += 256) {
        const int k = v >> 5, c = v & 31, h = h0 + c * 8;
        u32x4_t w = zero;
        if (k < rows && h < a.H) w = *reinterpret_cast<const u32x4_t*>((const bf16_t*)a.xs + (int64_t)k * a.H + h);
#pragma unroll
        for (int half = 0; half < 2; ++half) {          // four columns u of a group of 64: column 16 q + 4 j of them stands at 16 j + 4 q
            const int u = (c & 7) * 2 + half, at = (u & 3) * 4 + (u >> 2), ch = (c >> 3) * 8 + (at >> 1);
            *reinterpret_cast<uint2*>(xs + k * 512 + ((ch ^ swz(k, true)) << 4) + (at & 1) * 8) = half == 0 ? make_uint2(w.x, w.y) : make_uint2(w.z, w.w);
        }
    }
    u32x4_t e[KS];
    auto fetch = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < KS; ++u) {
            const int k = (tid >> 3) + 32 * u, col = t * DT_TILE + (tid & 7) * 8;
            e[u] = zero;
            if (k < rows && col < a.lde && t < end) e[u] = *reinterpret_cast<const u32x4_t*>((const bf16_t*)a.e + (int64_t)k * a.lde + col);
        }
    };
    fetch(first);
    __syncthreads();
    bf16x8_t fx[4][KS];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) fx[j][ks] = frag(xs, true, ks, wave * 64 + j * 16);
    __syncthreads();
    const int h = h0 + wave * 64 + g4 * 16;
    unsigned char* const stage = xs + 2 * ROWS * 128 + wave * 2048;
    for (int t = first; t < end; ++t) {
        unsigned char* s = xs + (t & 1) * (ROWS * 128);
#pragma unroll
        for (int u = 0; u < KS; ++u) {
            const int k = (tid >> 3) + 32 * u;
            *reinterpret_cast<u32x4_t*>(s + k * 128 + (((tid & 7) ^ swz(k, false)) << 4)) = e[u];
        }
        lds_barrier();
        fetch(t + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4_t acc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const bf16x8_t fe = frag(s, false, ks, i * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[j][ks], fe, acc[j], 0, 0, 0);
            }
            if constexpr (CF32) {
                const int c = t * DT_TILE + i * 16 + l16;
                if (c >= a.K) continue;
                float4* p = reinterpret_cast<float4*>((float*)a.out + (int64_t)c * a.H + h);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (h + 4 * j < a.H) {
                        const float4 b = p[j];
                        p[j] = make_float4(b.x + acc[j][0], b.y + acc[j][1], b.z + acc[j][2], b.w + acc[j][3]);
                    }
            } else {
                // by way of 2 KB of the wave's own to whole lines past the caches: what stays in the last one has to leave it under the next call's reading
                // of the table (64 rows, [128256, 4096]: this and that 193 + 257 us cached, 203 + 200 so; 16 rows, [50257, 2048] 37 + 54, 40 + 39)
#pragma unroll
                for (int j = 0; j < 4; j += 2)
                    *reinterpret_cast<u32x4_t*>(stage + l16 * 128 + (((2 * g4 + (j >> 1)) ^ (l16 & 7)) << 4)) =
                        u32x4_t{pack_bf16x2(acc[j][0], acc[j][1]), pack_bf16x2(acc[j][2], acc[j][3]), pack_bf16x2(acc[j + 1][0], acc[j + 1][1]),
                                pack_bf16x2(acc[j + 1][2], acc[j + 1][3])};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int r = half * 8 + (lane >> 3), c = t * DT_TILE + i * 16 + r, col = h0 + wave * 64 + (lane & 7) * 8;
                    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(stage + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
                    if (c < a.K && col < a.H) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_t*>((bf16_t*)a.out + (int64_t)c * a.H + col));
                }
            }
        }
    }
}

// ---- 5. dx -------------------------------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(256) void head_dx_sum_kernel(DxArgs a, const float* __restrict__ fac, const int32_t* __restrict__ y, T* __restrict__ dx) {
    constexpr int VN = Vec<T>::N;
    const int rows = live_rows(a.n_max, a.n_dev), vpr = a.H / VN;
    if (rows == 0) return;
    const DxPlan plan(rows, a.H, a.V, a.tile, a.resident);
    const int64_t total = (int64_t)rows * vpr;
    for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < total; v += (int64_t)gridDim.x * 256) {
        const int j = (int)(v / vpr), c = (int)(v - (int64_t)j * vpr) * VN;
        float s[VN];
        auto add = [&](const float* p) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < VN / 4; ++q) {
                const float4 w = reinterpret_cast<const float4*>(p)[q];
                s[4 * q] += w.x; s[4 * q + 1] += w.y; s[4 * q + 2] += w.z; s[4 * q + 3] += w.w;
            }
        };
#pragma unroll
        for (int e = 0; e < VN; ++e) s[e] = 0.f;
        add(a.slots + v * VN);
        if (plan.parts > 1) {
            const int tile = tile_number(j / a.tile, c / a.tile, plan.tm, plan.tn);
            if (tile >= plan.n_full) {
                const int64_t side = (int64_t)a.tile * a.tile;
                const float* p = a.more + plan.more(tile, 1, a.tile) + (j % a.tile) * a.tile + c % a.tile;
#pragma unroll 4
                for (int k = 1; k < plan.parts; ++k, p += side) add(p);
            }
        }
        const float f = fac[j];
        const bool live = y[j] >= 0;
#pragma unroll
        for (int e = 0; e < VN; ++e) s[e] = live ? f * s[e] : 0.f;
        Vec<T>::store(dx + v * VN, s);
    }
}

// ---- fp32 --------------------------------------------------------------------------------------------------
// The same steps with fp32 operands on the bf16 matrix cores: a value is the sum of three bf16 numbers, each the rounded rest of what is ahead of it, x = x1 + x2 + x3
// but for 2^-27 of x, and a product the sum of the six of the nine partial ones that are not below 2^-26 of it: x1 y1 + x1 y2 + x2 y1 + x2 y2 + x1 y3 + x3 y1, all in
// one fp32 accumulator.  That is fp32 accuracy at a sixth of the bf16 rate, 2.7 times that of the fp32 matrix instruction (values beyond 3.39e38 round to infinity).
// Tiles of 128x128, four waves of 64x64, steps of 32 k: operands go from memory to registers, a step ahead, and from there, split, to three planes in LDS; three
// blocks a CU cover each other's barriers.  MODE 0: A and B with k contiguous, 1: both k-major, 2: A contiguous, B k-major.  Planes of a k-contiguous operand are
// [row][32 k], 16-byte chunks XOR-ed with a function of the row that keeps the 16 lanes of one pass of a ds_read_b128 apart; of a k-major one [k][row], read
// transposed.  D = B-frag x A-frag: lane l holds row l % 16 and columns 4 * (l / 16) .. +3 of a fragment, as in the bf16 products.
// three blocks a CU at the price of a few spilled registers: logits 227 -> 208 us, the table's gradient 207 -> 193 (301 rows, [50257, 840])
#define F32_BOUNDS __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3)))
constexpr int F32_STEP = 32, F32_PLANE = 128 * F32_STEP * 2, F32_SMEM = 6 * F32_PLANE;

struct F32Tile {
    const float *A, *B;
    int64_t lda, ldb;
    int M, N;               // rows and columns that exist (MODE 1: of A's and B's columns)
    int k0, k1;             // the contraction's range
    int m0, n0;
};

// two values -> the rounded first, second and third parts of both
__device__ __forceinline__ void split2(float a, float b, unsigned& p1, unsigned& p2, unsigned& p3) {
    p1 = pack_bf16x2(a, b);
    a -= __uint_as_float(p1 << 16);
    b -= __uint_as_float(p1 & 0xFFFF0000u);
    p2 = pack_bf16x2(a, b);
    a -= __uint_as_float(p2 << 16);
    b -= __uint_as_float(p2 & 0xFFFF0000u);
    p3 = pack_bf16x2(a, b);
}

__device__ __forceinline__ int f32_swz(int row) { return -(row >> 2) & 3; }

template <int MODE> __device__ __forceinline__ void f32_tile(const F32Tile& t, unsigned char* smem, f32x4_t (&acc)[4][4]) {
    constexpr bool AK = MODE != 1, BK = MODE == 0;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1, l16 = lane & 15, g4 = lane >> 4;
    float4 ra[4], rb[4];
    // k contiguous: eight lanes a row of 32 k, rows 32 apart; k-major: 32 lanes a row of 128 columns, k 8 apart.  What does not exist lies outside a descriptor's
    // range: of the tile's rows, or of the step's k, which the scalar part of an address goes along
    constexpr unsigned OOB = 0x80000000u;
    auto lane_offset = [&](int base, int lim, int64_t ld, bool kc) __attribute__((always_inline)) {
        if (kc) return (unsigned)(tid >> 3) * (unsigned)ld * 4u + (tid & 7) * 16u;
        return base + (tid & 31) * 4 < lim ? (unsigned)(tid >> 5) * (unsigned)ld * 4u + (tid & 31) * 16u : OOB;
    };
    auto fetch = [&](float4 (&r)[4], const float* p, int64_t ld, int base, int lim, unsigned voff, int k, bool kc) __attribute__((always_inline)) {
        const int64_t at = kc ? (int64_t)base * ld : (int64_t)k * ld + base, have = kc ? min(lim - base, 128) * ld : (int64_t)max(0, min(t.k1 - k, F32_STEP)) * ld - base;
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p) + at, 0, (int)(have > 0 ? have * 4 : 0), 0x00020000);
        if (kc && k + (tid & 7) * 4 >= t.k1) voff = OOB;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[i] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(rs, voff + i * (kc ? 32u : 8u) * (unsigned)ld * 4u, kc ? k * 4 : 0, 0));
    };
    auto put = [&](const float4 (&r)[4], unsigned char* s, bool kc) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint2 p[3];
            split2(r[i].x, r[i].y, p[0].x, p[1].x, p[2].x);
            split2(r[i].z, r[i].w, p[0].y, p[1].y, p[2].y);
            int at;
            if (kc) {
                const int row = (tid >> 3) + 32 * i, ch = (tid & 7) >> 1;
                at = row * 64 + ((ch ^ f32_swz(row)) << 4) + (tid & 1) * 8;
            } else {
                const int k = (tid >> 5) + 8 * i, ch = (tid & 31) >> 1;
                at = k * 256 + ((ch ^ ((k & 3) << 2)) << 4) + (tid & 1) * 8;
            }
#pragma unroll
            for (int q = 0; q < 3; ++q) *reinterpret_cast<uint2*>(s + q * F32_PLANE + at) = p[q];
        }
    };
    // fragment f of the wave's 64 rows, plane q
    auto frag = [&](unsigned char* s, int w, int f, int q, bool kc) __attribute__((always_inline)) {
        s += q * F32_PLANE;
        if (kc) {
            const int row = w * 64 + f * 16 + l16;
            return *reinterpret_cast<const bf16x8_t*>(s + row * 64 + ((g4 ^ f32_swz(row)) << 4));
        }
        const int kl = 8 * g4 + (l16 >> 2), lc = (w * 64 + (f >> 1) * 32) / 8 + ((lane & 3) >> 1);
        unsigned char* p = s + kl * 256 + ((lc ^ ((kl & 3) << 2)) << 4) + (lane & 1) * 8 + (f & 1) * 32;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(__attribute__((address_space(3))) unsigned char*)p);
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(__attribute__((address_space(3))) unsigned char*)(p + 4 * 256));
        return __builtin_bit_cast(bf16x8_t, (s16x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (t.k0 >= t.k1) return;
    unsigned char *sa = smem, *sb = smem + 3 * F32_PLANE;
    const unsigned va = lane_offset(t.m0, t.M, t.lda, AK), vb = lane_offset(t.n0, t.N, t.ldb, BK);
    fetch(ra, t.A, t.lda, t.m0, t.M, va, t.k0, AK);
    fetch(rb, t.B, t.ldb, t.n0, t.N, vb, t.k0, BK);
    for (int k = t.k0; k < t.k1; k += F32_STEP) {
        lds_barrier();              // the step before has been read
        put(ra, sa, AK);
        put(rb, sb, BK);
        lds_barrier();
        // Nothing behind the last step.  One step ahead is enough with several blocks a CU (two, in 236 registers: dx 284 us for 225)
        fetch(ra, t.A, t.lda, t.m0, t.M, va, k + F32_STEP, AK);
        fetch(rb, t.B, t.ldb, t.n0, t.N, vb, k + F32_STEP, BK);
        CF_SCHED_FENCE();
        bf16x8_t fb[4][3];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 3; ++q) fb[j][q] = frag(sb, wn, j, q, BK);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf16x8_t fa[3];
#pragma unroll
            for (int q = 0; q < 3; ++q) fa[q] = frag(sa, wm, i, q, AK);
            // the smallest first; four accumulators in turn
            constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
            for (int z = 0; z < 6; ++z)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j][PB[z]], fa[PA[z]], acc[i][j], 0, 0, 0);
        }
    }
}

// What becomes of 16 rows' logits in a strip of columns from c on: lane l has row m = m0' + l % 16 and, in acc[j], columns c + 16 j + 4 * (l / 16) .. +3
template <int KIND> __device__ __forceinline__ void leave_f32(const HeadArgs& a, int rows, f32x4_t (&acc)[4], int m, int c, bool store) {
    const int g4 = (threadIdx.x & 63) >> 4;
    const float ref = m < rows ? a.ref[m] : INFINITY;
    const bool dead = ref == INFINITY;
    float s = 0.f, mx = -INFINITY, ey = 0.f;
    int y = -1;
    if (m < rows) { y = a.y[m]; ey = KIND == VALUES ? a.ey[m] : 0.f; }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int col = c + j * 16 + 4 * g4 + v;
            if (col >= a.V || (KIND == MAXIMA && col == y)) acc[j][v] = -INFINITY;
            mx = fmaxf(mx, acc[j][v]);
        }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * a.k;
    const float r = KIND == MAXIMA ? (mx == -INFINITY ? 0.f : mx) : ref;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int col = c + j * 16 + 4 * g4;
        float e[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            e[v] = __builtin_amdgcn_exp2f(fmaf(acc[j][v], a.k, -r));
            if (col + v == y) e[v] = ey;
            s += e[v];
            if (dead) e[v] = 0.f;
        }
        if (store && m < rows && col - a.c0 < a.lde)
            *reinterpret_cast<float4*>((float*)a.e + (int64_t)m * a.lde + (col - a.c0)) = make_float4(e[0], e[1], e[2], e[3]);
    }
    if (KIND != VALUES) {
        s += __shfl_xor(s, 16, 64);
        s += __shfl_xor(s, 32, 64);
        if (g4 == 0 && m < rows && c < a.V) {
            a.sums[(int64_t)(c / STRIP) * a.ldn + m] = KIND == MAXIMA ? mx + log2f(s) : s;
            if (KIND == SUMS && !dead && !(s <= FLAG_ABOVE)) a.flags[0] = a.flags[1 + (m >> 8)] = 1;
        }
    }
}

template <int KIND> __global__ F32_BOUNDS void head_logits_f32_kernel(HeadArgs a) {
    __shared__ __align__(16) unsigned char smem[F32_SMEM];
    if (a.flagged_only && a.flags[0] == 0) return;
    const int rows = live_rows(a.n_max, a.n_dev), tm = (rows + 127) / 128, tn = (a.c1 - a.c0 + 127) / 128;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    for (int64_t w = blockIdx.x; w < (int64_t)tm * tn; w += gridDim.x) {
        const int bm = (int)(w % tm), m0 = bm * 128, n0 = a.c0 + (int)(w / tm) * 128;
        if (a.flagged_only && a.flags[1 + (m0 >> 8)] == 0) continue;
        const F32Tile t{(const float*)a.x, (const float*)a.table, a.H, a.H, rows, min(a.c1, a.V), 0, a.H, m0, n0};
        f32x4_t acc[4][4];
        f32_tile<0>(t, smem, acc);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            leave_f32<KIND>(a, rows, acc[i], m0 + wm * 64 + i * 16 + (lane & 15), n0 + wn * 64, KIND != MAXIMA && n0 < a.store_end);
    }
}

// Fewer tiles than blocks that can be resident: a block takes a part of a tile's contraction and leaves its accumulators as they lie in its lanes; a wave a
// fragment row of a tile adds the parts up in order and does with the sum what the whole tile would.  A flagged tile is added up again, not multiplied.  The number of parts
// is that of the least cost: a step of 32 k takes 1.5, 2.1 or 2.6 us where one, two or three blocks share a CU, the second launch 3 us, 64 KB out and in 14 ns.
// Whole calls, no gradients, whole and in parts: 33 rows of [300, 8192] 453 and 45 us, 300 of [2500, 8192] 461 and 110, 1000 of [4096, 4096] (256 tiles) 242 and 190, 300
// of [12000, 2048] (282 tiles) 164 and 132, 600 of [4096, 512] 47 and 42; 1000 of [4096, 512] stays whole, 47 (in three parts 50).
struct F32Parts {
    int tiles, parts, per;          // per: steps a part; parts 1: whole tiles
    F32Parts(int n, int V, int H, int n_cu) {
        constexpr int64_t ns[4] = {0, 1500, 2100, 2600};
        const int steps = ceil_div(H, F32_STEP);
        tiles = (int)std::min<int64_t>((int64_t)ceil_div(n, 128) * ceil_div(V, 128), 1 << 24);
        parts = 1;
        int64_t best = tiles <= 3 * n_cu ? steps * ns[ceil_div(tiles, n_cu)] : 0;
        for (int p = 2; p * tiles <= 3 * n_cu && 4 * p <= steps; ++p) {
            const int64_t cost = ceil_div(steps, p) * ns[ceil_div(tiles * p, n_cu)] + 3000 + 14 * tiles * p;
            if (cost < best) { best = cost; parts = p; }
        }
        per = ceil_div(steps, parts);
        parts = ceil_div(steps, per);
    }
};
__global__ F32_BOUNDS void head_logits_part_f32_kernel(HeadArgs a, int tm, int tiles, int per) {
    __shared__ __align__(16) unsigned char smem[F32_SMEM];
    const int rows = live_rows(a.n_max, a.n_dev), tile = (int)blockIdx.x % tiles, part = (int)blockIdx.x / tiles, m0 = tile % tm * 128;
    if (m0 >= rows) return;
    const int k0 = part * per * F32_STEP;
    const F32Tile t{(const float*)a.x, (const float*)a.table, a.H, a.H, rows, a.V, k0, min(a.H, k0 + per * F32_STEP), m0, tile / tm * 128};
    f32x4_t acc[4][4];
    f32_tile<0>(t, smem, acc);
    f32x4_t* p = reinterpret_cast<f32x4_t*>(a.part) + (int64_t)blockIdx.x * 4096 + threadIdx.x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) p[(i * 4 + j) * 256] = acc[i][j];
}
template <int KIND> __global__ __launch_bounds__(64) void head_logits_join_f32_kernel(HeadArgs a, int tm, int tiles) {
    if (a.flagged_only && a.flags[0] == 0) return;
    const int rows = live_rows(a.n_max, a.n_dev), tile = (int)blockIdx.x >> 4, i = (int)blockIdx.x & 3, wave = ((int)blockIdx.x >> 2) & 3;
    const int m0 = tile % tm * 128, n0 = tile / tm * 128, m = m0 + (wave >> 1) * 64 + i * 16;
    if (m >= rows || n0 >= a.c1 || (a.flagged_only && a.flags[1 + (m0 >> 8)] == 0)) return;
    const f32x4_t* p = reinterpret_cast<const f32x4_t*>(a.part) + (int64_t)tile * 4096 + i * 1024 + wave * 64 + threadIdx.x;
    const int64_t step = (int64_t)tiles * 4096;
    f32x4_t acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    constexpr int U = 8;
    for (int q = 0; q < a.parts; q += U) {
        f32x4_t w[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) w[u][j] = p[min(q + u, a.parts - 1) * step + j * 256];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[j][v] += q + u < a.parts ? w[u][j][v] : 0.f;
    }
    leave_f32<KIND>(a, rows, acc, m + ((int)threadIdx.x & 15), n0 + (wave & 1) * 64, KIND != MAXIMA && n0 < a.store_end);
}

__global__ F32_BOUNDS void head_dx_f32_kernel(DxArgs a) {
    __shared__ __align__(16) unsigned char smem[F32_SMEM];
    const int rows = live_rows(a.n_max, a.n_dev);
    if (rows == 0) return;
    const DxPlan plan(rows, a.H, a.V, 128, a.resident);
    const int items = plan.items(), steps = (a.K + F32_STEP - 1) / F32_STEP;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    for (int w = blockIdx.x; w < items; w += gridDim.x) {
        int tile, part, bm, bn;
        plan.item(w, tile, part);
        tile_coords(tile, plan.tm, plan.tn, bm, bn);
        const int m0 = bm * 128, n0 = bn * 128, per = tile < plan.n_full ? steps : (steps + plan.parts - 1) / plan.parts, ld = part == 0 ? a.H : 128;
        float* const origin = part == 0 ? a.slots + (int64_t)m0 * a.H + n0 : a.more + plan.more(tile, part, 128);
        const F32Tile t{(const float*)a.e, (const float*)a.table, a.lde, a.H, rows, a.H, min(steps, part * per) * F32_STEP,
                        min(a.K, min(steps, part * per + per) * F32_STEP), m0, n0};
        f32x4_t acc[4][4];
        f32_tile<2>(t, smem, acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = wm * 64 + i * 16 + (lane & 15);
            if (m0 + r >= rows) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = wn * 64 + j * 16 + 4 * (lane >> 4);
                if (n0 + c >= a.H) continue;
                float4* p = reinterpret_cast<float4*>(origin + (int64_t)r * ld + c);
                float4 o = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
                if (!a.first) {
                    const float4 b = *p;
                    o.x += b.x; o.y += b.y; o.z += b.z; o.w += b.w;
                }
                *p = o;
            }
        }
    }
}

template <bool MAIN> __global__ F32_BOUNDS void head_dtable_f32_kernel(DtableArgs a) {
    __shared__ __align__(16) unsigned char smem[F32_SMEM];
    const int rows = live_rows(a.n_max, a.n_dev), tm = (a.K + 127) / 128, tn = (a.H + 127) / 128;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    for (int64_t w = blockIdx.x; w < (int64_t)tm * tn; w += gridDim.x) {
        const int m0 = (int)(w / tn) * 128, n0 = (int)(w % tn) * 128;
        const F32Tile t{(const float*)a.e, (const float*)a.xs, a.lde, a.H, a.lde, a.H, 0, rows, m0, n0};
        f32x4_t acc[4][4];
        f32_tile<1>(t, smem, acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = m0 + wm * 64 + i * 16 + (lane & 15);
            if (m >= a.K) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = n0 + wn * 64 + j * 16 + 4 * (lane >> 4);
                if (n >= a.H) continue;
                float4* p = reinterpret_cast<float4*>((float*)a.out + (int64_t)m * a.H + n);
                float4 o = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
                if (MAIN) {
                    const float4 b = *p;
                    o.x += b.x; o.y += b.y; o.z += b.z; o.w += b.w;
                }
                *p = o;
            }
        }
    }
}

// ---- fp32, few rows -----------------------------------------------------------------------------------
// The table's traffic counts, as for few bf16 rows, and is met with fp32 arithmetic (one row of [151936, 8192], 4.98 GB: logits 817 us, 6.1 TB/s, dx 775, the table's gradient 829; as
// products of tiles 3.8 ms in all): the logits by the fp32 matrix instruction (16x16x4; a lane's four adjacent k are four
// instructions, each with an accumulator of its own, so that a sum of H products has chains of H / 16), dx and the table's gradient, whose other operand is
// a few numbers, by fused multiply-adds.
// Up to how many rows: the logits (32 rows, [32000, 4096], 139 to 157 us, tiles 240; 64 rows, [50257, 2048], 187 and 177), the table's gradient, dx (16 rows, [50257, 2048], 871 and 146)
constexpr int F32_SUMS_FEW_ROWS = 32, F32_FEW_ROWS = 16, F32_DX_FEW_ROWS = 4;

template <int NF, int P> __global__ __launch_bounds__(512) void head_few_f32_kernel(HeadArgs a) {
    constexpr int R = P + 1, ROWS = 16 * NF, SLOT = ROWS * 256, TILE = 128;
    static_assert(NF <= 2, "a load of x a wave and step");
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float red[8][ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int rows = __builtin_amdgcn_readfirstlane(live_rows(a.n_max, a.n_dev)), H = a.H, steps = (H + 63) / 64;
    if (rows == 0) return;
    const int tiles = (a.V + TILE - 1) / TILE, rot = (int)(blockIdx.x * 37u) % steps;
    constexpr unsigned OOB = 0x80000000u;
    // x: four rows of 64 k a load, chunks of 16 bytes XOR-ed with the row; with few rows two waves load the same part
    const i32x4_t rx = make_rsrc(a.x, (int64_t)rows * H * 4);
    const int part = wave % (4 * NF), xrow = part * 4 + (lane >> 4), xk = ((lane ^ xrow) & 15) * 4;
    const unsigned xoff = (unsigned)xrow * (unsigned)H * 4u + xk * 4u, xdst = __builtin_amdgcn_readfirstlane(lds_addr_of(smem) + part * 1024);
    int lt = blockIdx.x, ls = 0, slot_in = 0;
    __amdgpu_buffer_rsrc_t rb;
    auto open = [&]() __attribute__((always_inline)) {
        const int64_t v0 = (int64_t)lt * TILE, have = lt < tiles ? min((int64_t)TILE, a.V - v0) : 0;
        rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>((const float*)a.table + (lt < tiles ? v0 : 0) * H), 0, (int)(have * H * 4), 0x00020000);
    };
    open();
    const unsigned boff = (unsigned)(wave * 16 + l16) * (unsigned)H * 4u + g4 * 16u;
    u32x4_t b[P][4];
    auto fetch = [&](u32x4_t (&to)[4]) __attribute__((always_inline)) {
        const int k0 = (ls + rot >= steps ? ls + rot - steps : ls + rot) * 64;
        dma16s(xdst + slot_in * SLOT, rx, k0 + xk < H ? xoff : OOB, (unsigned)k0 * 4u);
#pragma unroll
        for (int c = 0; c < 4; ++c) to[c] = __builtin_amdgcn_raw_buffer_load_b128(rb, k0 + c * 16 + g4 * 4 < H ? boff : OOB, (k0 + c * 16) * 4, 0);
        CF_SCHED_FENCE();
        slot_in = slot_in + 1 == R ? 0 : slot_in + 1;
        if (++ls == steps) {
            ls = 0;
            lt += (int)gridDim.x;
            open();
        }
    };
    float ref[NF], sum[NF];
    int y[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        ref[i] = i * 16 + l16 < rows ? a.ref[i * 16 + l16] : INFINITY;
        y[i] = i * 16 + l16 < rows ? a.y[i * 16 + l16] : -1;
        sum[i] = 0.f;
    }
#pragma unroll
    for (int p = 0; p < P; ++p) fetch(b[p]);
    f32x4_t acc[NF][4];
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int m = 0; m < 4; ++m) acc[i][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    int tile = blockIdx.x, s = 0, slot = 0;
    const int mine = (tiles - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
    for (int64_t left = (int64_t)mine * steps; left > 0; left -= P) {           // whole rounds, as for bf16
#pragma unroll
        for (int p = 0; p < P; ++p) {
            wait_vmcnt<(P - 1) * 5>();
            lds_barrier();
            const unsigned char* xs = smem + slot * SLOT + l16 * 256;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < NF; ++i) {
                    const f32x4_t fa = *reinterpret_cast<const f32x4_t*>(xs + i * 4096 + (((c * 4 + g4) ^ l16) << 4));
#pragma unroll
                    for (int m = 0; m < 4; ++m) acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b[p][c][m]), fa[m], acc[i][m], 0, 0, 0);
                }
            CF_SCHED_FENCE();
            fetch(b[p]);
            slot = slot + 1 == R ? 0 : slot + 1;
            if (++s == steps) {
                const int col = tile * TILE + wave * 16 + 4 * g4;
#pragma unroll
                for (int i = 0; i < NF; ++i) {
                    float e[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float l = (acc[i][0][v] + acc[i][1][v]) + (acc[i][2][v] + acc[i][3][v]);
                        e[v] = col + v < a.V && col + v != y[i] ? __builtin_amdgcn_exp2f(fmaf(l, a.k, -ref[i])) : 0.f;
                        sum[i] += tile < tiles ? e[v] : 0.f;
                        acc[i][0][v] = acc[i][1][v] = acc[i][2][v] = acc[i][3][v] = 0.f;
                    }
                    const int m = i * 16 + l16;
                    if (a.store_end > 0 && m < rows && tile < tiles && col < a.lde)
                        *reinterpret_cast<float4*>((float*)a.e + (int64_t)m * a.lde + col) =
                            ref[i] == INFINITY ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(e[0], e[1], e[2], e[3]);
                }
                s = 0;
                tile += (int)gridDim.x;
            }
        }
    }
    wait_vmcnt<0>();
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        sum[i] += __shfl_xor(sum[i], 16, 64);
        sum[i] += __shfl_xor(sum[i], 32, 64);
        if (g4 == 0) red[wave][i * 16 + l16] = sum[i];
    }
    __syncthreads();
    if ((int)threadIdx.x < rows) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += red[w][threadIdx.x];
        a.sums[(int64_t)blockIdx.x * a.ldn + threadIdx.x] = t;
        if (a.ref[threadIdx.x] != INFINITY && !(t <= FLAG_ABOVE)) a.flags[0] = a.flags[1] = 1;
    }
}

// what is the same for all threads, and not written during the kernel
__device__ __forceinline__ float uniform_load(const float* p) { return *(const __attribute__((address_space(4))) float*)(uintptr_t)p; }

// dx, split over the piece's rows of the table: split s of block's columns leaves [s][n_max, H] in the slots
template <int N> __global__ __launch_bounds__(256) void head_dx_few_f32_kernel(DxArgs a, int splits) {
    constexpr int U = 8;
    const int rows = live_rows(a.n_max, a.n_dev), hb = (a.H / 4 + 255) / 256, v = (int)blockIdx.x % hb * 256 + threadIdx.x, split = (int)blockIdx.x / hb;
    if (rows == 0 || v >= a.H / 4) return;
    const int per = (a.K + splits - 1) / splits, c0 = min(a.K, split * per), c1 = min(a.K, c0 + per);
    const float4* t = reinterpret_cast<const float4*>((const float*)a.table) + v;
    const int64_t ld = a.H / 4;
    float4 acc[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    auto take = [&](const float4& w, int c) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float e = uniform_load((const float*)a.e + (int64_t)min(j, rows - 1) * a.lde + c);
            acc[j].x = fmaf(e, w.x, acc[j].x); acc[j].y = fmaf(e, w.y, acc[j].y); acc[j].z = fmaf(e, w.z, acc[j].z); acc[j].w = fmaf(e, w.w, acc[j].w);
        }
    };
    int c = c0;
    for (; c + U <= c1; c += U) {
        float4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = t[(c + u) * ld];
#pragma unroll
        for (int u = 0; u < U; ++u) take(w[u], c + u);
    }
    for (; c < c1; ++c) take(t[c * ld], c);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (j >= rows) break;
        float4* p = reinterpret_cast<float4*>(a.slots + ((int64_t)split * a.n_max + j) * a.H) + v;
        if (!a.first) {
            const float4 o = *p;
            acc[j].x += o.x; acc[j].y += o.y; acc[j].z += o.z; acc[j].w += o.w;
        }
        *p = acc[j];
    }
}
__global__ __launch_bounds__(256) void head_dx_few_sum_f32_kernel(DxArgs a, int splits, const float* __restrict__ fac, const int32_t* __restrict__ y, float* __restrict__ dx) {
    const int rows = live_rows(a.n_max, a.n_dev), ld = a.H / 4, v = blockIdx.x * 256 + threadIdx.x;
    if (v >= rows * ld) return;
    const float4* p = reinterpret_cast<const float4*>(a.slots) + v;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 16
    for (int k = 0; k < splits; ++k) {
        const float4 w = p[(int64_t)k * a.n_max * ld];
        s.x += w.x; s.y += w.y; s.z += w.z; s.w += w.w;
    }
    const float f = fac[v / ld];
    const bool live = y[v / ld] >= 0;
    reinterpret_cast<float4*>(dx)[v] = live ? make_float4(f * s.x, f * s.y, f * s.z, f * s.w) : make_float4(0.f, 0.f, 0.f, 0.f);
}

template <int N, bool MAIN> __global__ __launch_bounds__(256) void head_dtable_few_f32_kernel(DtableArgs a, int per) {
    const int rows = live_rows(a.n_max, a.n_dev), hb = (a.H / 4 + 255) / 256, v = (int)blockIdx.x % hb * 256 + threadIdx.x, c0 = (int)blockIdx.x / hb * per;
    if (v >= a.H / 4 || (MAIN && rows == 0)) return;
    float4 x[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j < rows) x[j] = reinterpret_cast<const float4*>((const float*)a.xs + (int64_t)j * a.H)[v];
    }
    const int c1 = min(a.K, c0 + per);
#pragma unroll 2
    for (int c = c0; c < c1; ++c) {
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float e = rows > 0 ? uniform_load((const float*)a.e + (int64_t)min(j, rows - 1) * a.lde + c) : 0.f;
            o.x = fmaf(e, x[j].x, o.x); o.y = fmaf(e, x[j].y, o.y); o.z = fmaf(e, x[j].z, o.z); o.w = fmaf(e, x[j].w, o.w);
        }
        float4* p = reinterpret_cast<float4*>((float*)a.out + (int64_t)c * a.H) + v;
        if constexpr (MAIN) {
            const float4 b = *p;
            *p = make_float4(b.x + o.x, b.y + o.y, b.z + o.z, b.w + o.w);
        } else {
            __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, o), reinterpret_cast<u32x4_t*>(p));
        }
    }
}

// ---- workspace and launches --------------------------------------------------------------------------------

struct HeadWs {
    int strips, ldn, tile, resident, cap;       // of dx: a tile's rows and columns, blocks that are resident at a time.  cap: columns of e (0: too little room, or no gradient)
    size_t ref, a, ey, y, terms, flags, sums, xs, slots, more, part, e, total;
    HeadWs(int V, int H, int n_rows, int dtype, bool need_dx, bool need_dt, size_t bytes) {
        const int n = n_rows > 0 ? n_rows : 1;
        const size_t es = dtype_size(dtype);
        strips = ceil_div(V, STRIP);
        ldn = (int)align_up((size_t)n, 16);
        size_t at = 0;
        auto take = [&](size_t b) { const size_t p = at; at += align_up(b, 256); return p; };
        ref = take((size_t)n * 4);
        a = take((size_t)n * 4);
        ey = take((size_t)n * 4);
        y = take((size_t)n * 4);
        terms = take((size_t)n * 16);
        flags = take((size_t)(ceil_div(n, 256) + 1) * 4);
        sums = take((size_t)(n <= FEW_ROWS ? std::max(strips, compute_units()) : strips) * ldn * 4);
        xs = take(need_dt ? (size_t)n * H * es : 0);
        tile = dtype == CF_F32 || n <= 128 ? 128 : 256;
        resident = compute_units() * (dtype == CF_F32 ? 3 : 1);
        slots = take(need_dx ? (size_t)n * H * 4 : 0);
        more = take(need_dx ? (size_t)2 * resident * tile * tile * 4 : 0);         // at most two rounds of parts
        // fp32 logits in parts, at most three a CU: gone before dx begins
        const F32Parts P(n, V, H, compute_units());
        part = need_dx ? more : take(dtype == CF_F32 && n > F32_SUMS_FEW_ROWS && P.parts > 1 ? (size_t)P.tiles * P.parts * 65536 : 0);
        e = at;
        cap = 0;
        total = at;
        if (!need_dx && !need_dt) return;
        int64_t whole = (int64_t)align_up((size_t)V, 256), least = std::min<int64_t>(whole, 2048), most = whole;
        if (dtype == CF_F32) {      // 32-bit offsets within a tile's 128 rows
            most = std::min<int64_t>(most, 1 << 21);
            least = std::min(least, most);
        } else {                    // matrices below 2 GiB: 32-bit offsets
            const int64_t lim = ((int64_t)1 << 31) - 1;
            most = std::min({most, lim / (2 * (std::max<int64_t>(n, 256) + 64)) / 256 * 256, (lim / (2 * (int64_t)H) - 256) / 256 * 256});
            least = std::min(least, most);
        }
        if (most < 256) { cap = -1; return; }
        int64_t c = bytes > at ? (int64_t)((bytes - at) / ((size_t)n * es)) / 256 * 256 : 0;
        cap = (int)std::max(least, std::min(most, c));
        total = at + align_up((size_t)n * cap * es, 256);
    }
};

template <typename T> static void launch_dx_sum(const DxArgs& a, const float* fac, const int32_t* y, void* dx, hipStream_t st) {
    const int64_t vecs = (int64_t)a.n_max * (a.H / Vec<T>::N);
    head_dx_sum_kernel<T><<<(int)std::min<int64_t>((vecs + 255) / 256, 32 * compute_units()), 256, 0, st>>>(a, fac, y, (T*)dx);
}

template <typename T> struct HeadLaunch;
template <> struct HeadLaunch<bf16_t> {
    template <int KIND> static hipError_t logits(const HeadArgs& a, hipStream_t st) {
        static std::atomic<uint64_t> lds_ok{0};
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&head_logits_kernel<KIND>), GEMM_SMEM, lds_ok);
        if (e != hipSuccess) return e;
        head_logits_kernel<KIND><<<compute_units(), 256, GEMM_SMEM, st>>>(a);
        return hipGetLastError();
    }
    template <int NF> static hipError_t few(const HeadArgs& a, hipStream_t st) {
        static std::atomic<uint64_t> lds_ok{0};
        constexpr int P = NF > 4 ? 6 : 8, lds = (P + 1) * NF * 16 * 128 + NF * 16 * 256;
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&head_few_kernel<NF, P>), lds, lds_ok);
        if (e != hipSuccess) return e;
        head_few_kernel<NF, P><<<a.strips, 512, lds, st>>>(a);
        return hipGetLastError();
    }
    static hipError_t dx_sum(const DxArgs& a, const float* fac, const int32_t* y, bf16_t* dx, hipStream_t st) {
        launch_dx_sum<bf16_t>(a, fac, y, dx, st);
        return hipGetLastError();
    }
    // sums of the whole vocabulary; sets the number of sums a row has
    static hipError_t sums(HeadArgs& a, hipStream_t st) {
        if (a.n_max > FEW_ROWS) return logits<SUMS>(a, st);
        a.strips = few_blocks(a.V, compute_units());
        return a.n_max <= 16 ? few<1>(a, st) : a.n_max <= 32 ? few<2>(a, st) : a.n_max <= 64 ? few<4>(a, st) : few<8>(a, st);
    }
    static hipError_t dx(const DxArgs& a, hipStream_t st) {
        static std::atomic<uint64_t> lds_ok{0};
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&head_dx_kernel), GEMM_SMEM, lds_ok);
        if (e != hipSuccess) return e;
        head_dx_kernel<<<a.resident, 256, GEMM_SMEM, st>>>(a);
        return hipGetLastError();
    }
    template <int KS> static hipError_t dtable_few(const DtableArgs& a, bool main, hipStream_t st) {
        const int hb = ceil_div(a.H, 256), tiles = ceil_div(a.K, DT_TILE), per = ceil_div(tiles, std::max(1, 8 * compute_units() / hb)), grid = hb * ceil_div(tiles, per);
        if (main) head_dtable_few_kernel<KS, true><<<grid, 256, 0, st>>>(a, per);
        else head_dtable_few_kernel<KS, false><<<grid, 256, 0, st>>>(a, per);
        return hipGetLastError();
    }
    static hipError_t dtable(DtableArgs a, bool main, hipStream_t st) {
        if (a.n_max <= DT_FEW_ROWS) return a.n_max <= 32 ? dtable_few<1>(a, main, st) : a.n_max <= 64 ? dtable_few<2>(a, main, st) : dtable_few<4>(a, main, st);
        static std::atomic<uint64_t> lds_ok[2];
        void (*const kernel)(DtableArgs) = main ? head_dtable_kernel<true> : head_dtable_kernel<false>;
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), GEMM_SMEM, lds_ok[main]);
        if (e != hipSuccess) return e;
        const int tiles = ceil_div(a.K, 256) * ceil_div(a.H, 256);
        plan_tiles(tiles, compute_units(), a.n_full, a.sub);
        kernel<<<std::min(a.n_full + (tiles - a.n_full) * a.sub, compute_units()), 256, GEMM_SMEM, st>>>(a);
        return hipGetLastError();
    }
};
template <> struct HeadLaunch<float> {
    static int grid(int64_t items) { return (int)std::min<int64_t>(items, MAX_GRID); }
    // of the launch's columns, or of the flagged tiles, whose parts are still there
    template <int KIND> static hipError_t logits(const HeadArgs& a, hipStream_t st) {
        if (a.parts > 1 && a.flagged_only) return join<KIND>(a, st);
        head_logits_f32_kernel<KIND><<<grid((int64_t)ceil_div(a.n_max, 128) * ceil_div(a.c1 - a.c0, 128)), 256, 0, st>>>(a);
        return hipGetLastError();
    }
    template <int KIND> static hipError_t join(const HeadArgs& a, hipStream_t st) {
        const int tm = ceil_div(a.n_max, 128), tiles = tm * ceil_div(a.V, 128);
        head_logits_join_f32_kernel<KIND><<<16 * tiles, 64, 0, st>>>(a, tm, tiles);
        return hipGetLastError();
    }
    static hipError_t sums(HeadArgs& a, hipStream_t st) {
        if (a.n_max > F32_SUMS_FEW_ROWS) {
            const F32Parts P(a.n_max, a.V, a.H, compute_units());
            a.parts = P.parts;
            if (P.parts == 1) return logits<SUMS>(a, st);
            head_logits_part_f32_kernel<<<P.tiles * P.parts, 256, 0, st>>>(a, ceil_div(a.n_max, 128), P.tiles, P.per);
            const hipError_t e = hipGetLastError();
            return e != hipSuccess ? e : join<SUMS>(a, st);
        }
        a.strips = few_blocks(a.V, compute_units());
        return a.n_max <= 16 ? few<1>(a, st) : few<2>(a, st);
    }
    template <int NF> static hipError_t few(const HeadArgs& a, hipStream_t st) {
        static std::atomic<uint64_t> lds_ok{0};
        constexpr int P = 6, lds = (P + 1) * NF * 16 * 256;
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&head_few_f32_kernel<NF, P>), lds, lds_ok);
        if (e != hipSuccess) return e;
        head_few_f32_kernel<NF, P><<<a.strips, 512, lds, st>>>(a);
        return hipGetLastError();
    }
    // parts of dx's sum over the vocabulary: eight blocks a CU, each with as much to read as it leaves, in the slots there are
    static int splits(const DxArgs& a) {
        const int hb = ceil_div(a.H / 4, 256);
        const int64_t room = ((int64_t)a.n_max * a.H + (int64_t)2 * a.resident * a.tile * a.tile) / ((int64_t)a.n_max * a.H);
        return (int)std::max<int64_t>(1, std::min({(int64_t)8 * compute_units() / hb, room, (int64_t)a.V / (16 * a.n_max)}));
    }
    static hipError_t dx_sum(const DxArgs& a, const float* fac, const int32_t* y, float* dx, hipStream_t st) {
        if (a.n_max <= F32_DX_FEW_ROWS) head_dx_few_sum_f32_kernel<<<ceil_div((int64_t)a.n_max * (a.H / 4), 256), 256, 0, st>>>(a, splits(a), fac, y, dx);
        else launch_dx_sum<float>(a, fac, y, dx, st);
        return hipGetLastError();
    }
    static hipError_t dx(const DxArgs& a, hipStream_t st) {
        if (a.n_max <= F32_DX_FEW_ROWS) {
            const int s = splits(a), g = s * ceil_div(a.H / 4, 256);
            if (a.n_max <= 1) head_dx_few_f32_kernel<1><<<g, 256, 0, st>>>(a, s);
            else head_dx_few_f32_kernel<4><<<g, 256, 0, st>>>(a, s);
            return hipGetLastError();
        }
        head_dx_f32_kernel<<<2 * a.resident, 256, 0, st>>>(a);
        return hipGetLastError();
    }
    template <int N> static hipError_t dtable_few(const DtableArgs& a, bool main, hipStream_t st) {
        const int hb = ceil_div(a.H / 4, 256), per = ceil_div(a.K, std::max(1, 16 * compute_units() / hb)), g = hb * ceil_div(a.K, per);
        if (main) head_dtable_few_f32_kernel<N, true><<<g, 256, 0, st>>>(a, per);
        else head_dtable_few_f32_kernel<N, false><<<g, 256, 0, st>>>(a, per);
        return hipGetLastError();
    }
    static hipError_t dtable(const DtableArgs& a, bool main, hipStream_t st) {
        if (a.n_max <= F32_FEW_ROWS) return a.n_max <= 1 ? dtable_few<1>(a, main, st) : a.n_max <= 4 ? dtable_few<4>(a, main, st) : dtable_few<16>(a, main, st);
        const int g = grid((int64_t)ceil_div(a.K, 128) * ceil_div(a.H, 128));
        if (main) head_dtable_f32_kernel<true><<<g, 256, 0, st>>>(a);
        else head_dtable_f32_kernel<false><<<g, 256, 0, st>>>(a);
        return hipGetLastError();
    }
};

#define CF_TRY(call)                            \
    do {                                        \
        const hipError_t e_ = (call);           \
        if (e_ != hipSuccess) return e_;        \
    } while (0)

template <typename T>
static hipError_t launch_head(HeadArgs a, LossArgs l, const HeadWs& L, unsigned char* ws, void* dx, void* dtable, bool main, float* stats, hipStream_t st) {
    const int n = a.n_max, V = a.V, H = a.H;
    if (n > 0) {
        const bool grads = dx != nullptr || dtable != nullptr;
        a.ref = (float*)(ws + L.ref);
        a.a = (float*)(ws + L.a);
        a.ey = (float*)(ws + L.ey);
        a.y = (int32_t*)(ws + L.y);
        a.flags = (int32_t*)(ws + L.flags);
        a.sums = (float*)(ws + L.sums);
        a.ldn = L.ldn;
        a.strips = L.strips;
        l.terms = (float4*)(ws + L.terms);
        void* xs = dtable != nullptr ? ws + L.xs : nullptr;
        const int first = std::min(V, L.cap);           // columns whose exponentials are kept
        a.c0 = 0; a.c1 = V; a.lde = (int)align_up((size_t)first, 8); a.store_end = grads ? first : 0; a.e = grads ? ws + L.e : nullptr;
        a.flagged_only = false;
        a.part = (float*)(ws + L.part);
        a.parts = 1;
        const int blocks = ceil_div(n, 4);
        head_rows_kernel<T><<<std::min(blocks, 8 * compute_units()), 256, 0, st>>>(a, l);
        CF_TRY(hipGetLastError());
        CF_TRY(HeadLaunch<T>::sums(a, st));
        a.flagged_only = true;
        CF_TRY(HeadLaunch<T>::template logits<MAXIMA>(a, st));
        head_finish_kernel<T><<<ceil_div(n, 16), 1024, 0, st>>>(a, l, xs, n <= 16 ? stats : nullptr);
        CF_TRY(hipGetLastError());
        DxArgs d{};
        for (int c = 0; grads && c < V; c += L.cap) {
            const int w = std::min(L.cap, V - c);
            a.c0 = c; a.c1 = c + w; a.lde = (int)align_up((size_t)w, 8); a.store_end = c + w; a.flagged_only = c == 0;
            CF_TRY(HeadLaunch<T>::template logits<VALUES>(a, st));
            if (dx != nullptr)
                CF_TRY(HeadLaunch<T>::dx(d = DxArgs{a.e, (const T*)a.table + (int64_t)c * H, a.lde, w, H, n, a.n_dev, (float*)(ws + L.slots), (float*)(ws + L.more), V, L.tile,
                                                    L.resident, c == 0}, st));
            if (dtable != nullptr)
                CF_TRY(HeadLaunch<T>::dtable(DtableArgs{a.e, xs, (char*)dtable + (int64_t)c * H * (main ? 4 : (int)sizeof(T)), a.lde, w, H, n, a.n_dev, 0, 1}, main, st));
        }
        if (dx != nullptr) CF_TRY(HeadLaunch<T>::dx_sum(d, a.a, a.y, (T*)dx, st));
    } else if (dtable != nullptr && !main) {
        CF_TRY(launch_fill_zero(dtable, (size_t)V * H * sizeof(T), st));
    }
    if (stats != nullptr && (n == 0 || n > 16)) launch_loss_stats((const float4*)(ws + L.terms), n, a.n_dev, l.norm, stats, st);
    return hipGetLastError();
}

}  // namespace cf

using namespace cf;

static cf_status head_sizes(const cf_loss_desc* d, int32_t H, int32_t max_kept) {
    if (!d) return CF_ERR_NULL;
    if (d->dtype != CF_BF16 && d->dtype != CF_F32) return CF_ERR_DTYPE;
    if (d->V <= 0 || d->V > (1 << 30) || H <= 0 || H % (d->dtype == CF_F32 ? 4 : 8) != 0 || max_kept < 0 || max_kept > (1 << 30)) return CF_ERR_SHAPE;
    // tiles, and threads of a launch, are counted in 32 bits
    if (H > (1 << 20) || max_kept > (1 << 22) || (int64_t)ceil_div(max_kept, 256) * ceil_div(d->V, 256) >= (1 << 29)) return CF_ERR_UNSUPPORTED;
    if (d->dtype == CF_BF16 && (int64_t)max_kept * H * 2 >= ((int64_t)1 << 31)) return CF_ERR_UNSUPPORTED;
    return CF_OK;
}

extern "C" {

size_t cf_head_loss_workspace_bytes(const cf_loss_desc* desc, int32_t H, int32_t max_kept, int32_t need_dx, int32_t need_dtable, size_t limit) {
    if (head_sizes(desc, H, max_kept) != CF_OK) return 0;
    const HeadWs L(desc->V, H, max_kept, desc->dtype, need_dx != 0, need_dtable != 0, limit);
    return L.cap < 0 ? 0 : L.total;
}

cf_status cf_head_loss(const cf_loss_desc* desc, int32_t H, const void* x_kept, const void* table, const int64_t* targets, const float* old_logp,
                       const float* ref_logp, const float* advantages, const float* weights, const int32_t* idx, const int32_t* n_kept_dev,
                       int32_t max_kept, void* dx_kept, void* dtable, int32_t main_grad, float* logp, float* stats, void* ws, size_t ws_bytes,
                       cf_stream stream) {
    if (!desc || !x_kept || !table || !targets) return CF_ERR_NULL;
    if (!dx_kept && !dtable && !logp && !stats) return CF_ERR_NULL;
    cf_status ok = loss_desc_check(desc, old_logp, ref_logp, advantages, max_kept);
    if (ok == CF_OK) ok = head_sizes(desc, H, max_kept);
    if (ok != CF_OK) return ok;
    if (main_grad != 0 && main_grad != 1) return CF_ERR_SHAPE;
    if (off_by(x_kept, 16) || off_by(table, 16) || off_by(dx_kept, 16) || off_by(dtable, 16) || off_by(targets, 8)) return CF_ERR_SHAPE;
    for (const void* p : {(const void*)old_logp, (const void*)ref_logp, (const void*)advantages, (const void*)weights, (const void*)idx,
                          (const void*)n_kept_dev, (const void*)logp, (const void*)stats})
        if (off_by(p, 4)) return CF_ERR_SHAPE;
    const uint64_t es = dtype_size(desc->dtype), xb = (uint64_t)max_kept * H * es, tb = (uint64_t)desc->V * H * es;
    const uint64_t db = (uint64_t)desc->V * H * (main_grad ? 4 : es);
    if ((dx_kept != x_kept && ranges_meet(dx_kept, xb, x_kept, xb)) || ranges_meet(dx_kept, xb, table, tb) || ranges_meet(dtable, db, table, tb) ||
        ranges_meet(dtable, db, x_kept, xb) || ranges_meet(dtable, db, dx_kept, xb))
        return CF_ERR_SHAPE;
    const HeadWs L(desc->V, H, max_kept, desc->dtype, dx_kept != nullptr, dtable != nullptr, ws_bytes);
    if (L.cap < 0) return CF_ERR_UNSUPPORTED;
    if (!ws || off_by(ws, 256) || ws_bytes < L.total) return CF_ERR_WORKSPACE;
    const LossArgs l = loss_args(desc, targets, old_logp, ref_logp, advantages, weights, idx, n_kept_dev, max_kept, logp);
    HeadArgs a{};
    a.x = x_kept; a.table = table; a.H = H; a.V = desc->V; a.n_max = max_kept; a.n_dev = n_kept_dev; a.k = l.k;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    unsigned char* w = (unsigned char*)ws;
    const hipError_t e = desc->dtype == CF_F32 ? launch_head<float>(a, l, L, w, dx_kept, dtable, main_grad != 0, stats, st)
                                               : launch_head<bf16_t>(a, l, L, w, dx_kept, dtable, main_grad != 0, stats, st);
    return e == hipSuccess ? CF_OK : CF_ERR_HIP;
}

}  // extern "C"
