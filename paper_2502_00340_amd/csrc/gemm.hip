// Dimension-reduced dense GEMMs (Sec. 3.2): next-node gradient dX = dY * W^T and
// parameter gradient dW = X^T * dY on kept rows only.
//
//   mode NT: C[M,N] = sum_seg A[M,K] * B[N,K]^T   (both operands contiguous along K)
//   mode TN: C[M,N] = sum_seg A[K,M]^T * B[K,N]   (both operands contiguous along M / N;
//                                                  K is the kept-token dimension)
// Up to six (A, B, K) segments accumulate into one output tile, which sums
// the gradients of a tensor consumed by several linears without rounding in
// between (e.g. d_gate*Wg^T + d_up*Wu^T).
//
// bf16 path: 16x16x32 bf16 MFMA, fp32 accumulators, 256 threads = 2x2 waves, one
// block per CU.  The block tile is (64*TM) x (64*TN) with wave tiles of
// (32*TM) x (32*TN); three shapes are compiled into one kernel: 256x256 (the
// wave tile with the fewest LDS bytes per MFMA), 256x128 and 128x128; the NT kernel
// also has 256x192, for outputs whose 256x256 tiles would leave CUs idle (a dX of
// 4096 x 3072 is 16 x 12 = 192 such tiles but 16 x 16 = 256 of the narrower ones).
//   * Why the small MFMA.  Under these kernels the chip is power-limited: the shader clock
//     settles at 1.5-1.9 GHz instead of 2.4, and 128 CUs deliver 75 % of what 256 do.
//     What counts is therefore energy per flop, not only cycles: 16x16x32 reads and writes
//     its accumulators half as often per flop as 32x32x16 does, runs at a 14 % higher
//     clock for the same work and gains 3-6 % on the large products, although its
//     16-cycle issue rhythm leaves less room for the other instructions (the matrix
//     cores are busy 72 % of the cycles instead of 77 %).  Fragment reads from LDS cost
//     no cycles any more but about 9 % of the clock.
//   * Tile scheduling.  A launch has as many blocks as CUs; a block walks through its
//     share of the output tiles.  The 256x256 tiles that fill whole rounds of the CUs
//     come first; the tiles of the last, partial round are cut into 2 or 4 sub-tiles
//     when that shortens the tail (a 3.5-round problem takes 3 rounds of full tiles
//     and one of half tiles instead of 4 rounds).  Within each group the 8 XCDs (block
//     id mod 8) take contiguous runs of a band-major tile order, so the blocks resident
//     on one XCD share operand panels in that XCD's L2.  Between two tiles of a block
//     the loads of the next tile's first K-steps are already in flight while the
//     finished tile leaves, and its stores drain under the next tile's MFMAs (the
//     write-out of a tile used to be 13 % of its time).
//   * Operand tiles move in K-steps of 32 through a ring of four 32 KB LDS stages (the 128x128
//     tile: eight of 16 KB, four pairs instead of two, three of them ahead),
//     filled by buffer_load ... lds (16 bytes per lane, no register hop).  K-steps are
//     handled in pairs (64 k: one whole 128-byte line of every NT operand row, eight such
//     lines per load); a pair is loaded two pairs ahead, into the two
//     stages that the barrier of the pair being computed has just retired; completion
//     is tracked with vmcnt.  Ragged edges come from the buffer descriptor's range
//     check, which returns zeros, so there are no branches around loads.
//   * One LDS barrier per 64 K.  A pair is 2*TM sub-steps: one 32-row block of the
//     wave's A rows against all its B columns for one K-step (16 MFMAs in a 128x128 wave
//     tile).  The A fragments of the next sub-step and a share of the B fragments of
//     the next K-step are read ahead of their use, and the instruction stream is laid
//     out by hand: a gap between two MFMAs carries at most one fragment read and one
//     instruction of a load (the write of M0 goes ahead of an MFMA, the load behind it).
//     The loop body is two pairs, which makes every stage a compile-time constant: an
//     LDS read is a loop-invariant per-lane base register plus an instruction offset, a
//     load takes its per-lane offset from a register that is fixed for the whole K
//     segment and its K position from the instruction's scalar offset, so the steady
//     state has no vector ALU instruction besides the MFMAs.
//   * The loads of a pair go out in groups spread over the sub-steps (four groups in
//     NT, three in TN; two cost 4 %): a CU sustains only so many bytes in flight, and a
//     burst of 64 KB stalls the stream.
//   * NT pair: [rows][64 k], 128-byte rows, the 16-byte chunk index of a row XOR-ed with a
//     function of the row chosen so that the 16 lanes that the LDS serves in one pass of a
//     ds_read_b128 hit distinct banks (see nt_swz); a lane of the loading wave picks the
//     global chunk that belongs in its (fixed) LDS slot.
//   * TN stage: [32 k][rows] exactly as in memory, with the 64-byte group index of a
//     k-row XOR-ed with k%4; fragments come out of LDS through the transpose read
//     (ds_read_b64_tr_b16), in the same register layout as the NT ones, so MFMA
//     order and epilogue are shared.  The four k-rows that a group of 16 lanes touches
//     in one transpose read land in four different 64-byte bank groups.
//   * The MFMA is issued with the operands swapped (D = B-frag x A-frag), so a lane
//     ends up with 4 adjacent output columns of one row; the epilogue packs them to
//     bf16 and sends them, 32 rows of the wave tile at a time, through 8 KB of LDS of
//     the wave's own (above the operand stages, which the next tile is filling by
//     then) to full-row 16-byte stores.
// fp32 path (check mode): plain LDS-tiled FMA kernel.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "gemm_tiles.h"
#include "mfma_util.h"

namespace cf {

// Mode TN: up to TN_MAX products C_j [M_j,N_j] = A_j^T * B_j over the same K rows (A, B, C, M and N above are unused).  Their
// tiles form one list, product by product; all the parameter gradients of a layer are one launch, whose tiles fill whole
// rounds of the CUs but for one remainder, where a launch per product has a remainder each: [8192 rows, H = 2048,
// F = 5632, 32/4 heads of 64] 176 + 352 + 64 + 80 tiles are 2.6 rounds instead of 1 + 2 + 1 + 1, into fp32 buffers 822 us in
// four launches and 750 in one; [841 rows, H = 4096, F = 1792, 4/1 heads of 128] 81 us in four, 60 in one.
struct TnArgs : GemmArgs {
    GemmTnProb p[TN_MAX];
    int end[TN_MAX];    // tiles of products 0..j
    int n_blocks;       // blocks that walk through the tiles; those behind them sum the gain gradients up
    GainGrads gain;
};

__global__ __launch_bounds__(256) void gemm_nt_kernel(GemmArgs g) {
    extern __shared__ __align__(16) unsigned char smem[];
    int Mx = g.M, n_full = g.n_full, sub = g.sub, tile_n = g.tile_n;
    if (g.n_dev != nullptr) {
        // the kept-token count is a device value: clamp the rows to it and plan the tiles here, as the host does for sizes it
        // knows (the output shape depends on it)
        int n = *g.n_dev;
        n = __builtin_amdgcn_readfirstlane(n < 0 ? 0 : n);
        Mx = n < Mx ? n : Mx;
        plan_launch(Mx, g.N, (int)gridDim.x, n_full, sub, tile_n);
        n_full = __builtin_amdgcn_readfirstlane(n_full);
        sub = __builtin_amdgcn_readfirstlane(sub);
        tile_n = __builtin_amdgcn_readfirstlane(tile_n);
    }
    const TileRef whole{0, 0, Mx, g.N, g.A[0], g.B[0], g.C};
    int per = 0;
    const int parts = g.parts.count(Mx, per);
    if (__builtin_expect(parts > 1, 0)) {
        // An item is a part of a 128x128 tile.  The items of one part come together, column of tiles by column: an XCD's share
        // of them reads the same rows of A and B.
        const int tm = (Mx + 127) / 128, tiles = tm * ((g.N + 127) / 128), items = tiles * parts;
        if ((int)blockIdx.x >= items) return;
        const int w = xcd_order((int)blockIdx.x, items);
        const int part = __builtin_amdgcn_readfirstlane(w / tiles), tile = __builtin_amdgcn_readfirstlane(w % tiles);
        TileRef t = whole;
        t.m0 = __builtin_amdgcn_readfirstlane((tile % tm) * 128);
        t.n0 = __builtin_amdgcn_readfirstlane((tile / tm) * 128);
        per = __builtin_amdgcn_readfirstlane(per);
        gemm_tiles<0, 2, 2, true, false>(g, g.K[0], t, [](TileRef&) { return false; }, smem, part * per,
                                         min(g.parts.pairs, part * per + per), g.parts.slots + ((int64_t)tile * parts + part) * (128 * 128));
        return;
    }
    const int tiles_m = (Mx + 255) / 256, tiles_n = (g.N + 255) / 256;
    if (tile_n == 192) {
        // tiles of 256x192, all of one kind: block b takes tiles b, b + gridDim.x, ...
        const int tiles_n192 = (g.N + 191) / 192, n_items = tiles_m * tiles_n192;
        int w = (int)blockIdx.x;
        // with a device-side count there are as many blocks as CUs, whatever the number of tiles: a block
        // past the last tile would compute another block's tile a second time
        if (w >= n_items) return;
        auto tile = [&](int w, TileRef& t) __attribute__((always_inline)) {
            int bm, bn;
            tile_coords(xcd_order(w, n_items), tiles_m, tiles_n192, bm, bn);
            t = whole;
            t.m0 = __builtin_amdgcn_readfirstlane(bm * 256);
            t.n0 = __builtin_amdgcn_readfirstlane(bn * 192);
        };
        TileRef t;
        tile(w, t);
        gemm_tiles<0, 4, 3, false, false>(g, g.K[0], t, [&](TileRef& nx) __attribute__((always_inline)) {
            w += (int)gridDim.x;
            if (w >= n_items) return false;
            tile(w, nx);
            return true;
        }, smem);
        return;
    }
    gemm_items<0, false>(g, g.K[0], tiles_m * tiles_n, n_full, sub, (int)gridDim.x, [&](int l, TileRef& t, int& bm, int& bn) __attribute__((always_inline)) {
        t = whole;
        tile_coords(l, tiles_m, tiles_n, bm, bn);
    }, smem);
}

// CF32: C is fp32 (main-gradient buffers) and the products are added to it without rounding.
template <bool CF32>
__global__ __launch_bounds__(256) void gemm_tn_kernel(TnArgs g) {
    extern __shared__ __align__(16) unsigned char smem[];
    // Blocks behind those of the tiles sum the gain gradients up: where a CU has no tile left in the last, partial round they cost
    // nothing, where a launch of their own is 5 us ([841 of 2103 rows, H = 4096, F = 1792, 4/1 heads] layer call 231.0 and 226.3 us).
    if ((int)blockIdx.x >= g.n_blocks) {
        using T = std::conditional_t<CF32, float, bf16_t>;
        gain_grads_block<T, CF32>(g.gain, (int)blockIdx.x - g.n_blocks, reinterpret_cast<float (*)[33]>(smem));
        return;
    }
    int K0x = g.K[0];
    if (g.n_dev != nullptr) {           // the contraction is over the kept tokens: only its length depends on the count
        int n = *g.n_dev;
        n = __builtin_amdgcn_readfirstlane(n < 0 ? 0 : n);
        K0x = n < K0x ? n : K0x;
    }
    gemm_items<1, CF32>(g, K0x, g.end[TN_MAX - 1], g.n_full, g.sub, g.n_blocks, [&](int l, TileRef& t, int& bm, int& bn) __attribute__((always_inline)) {
        int j = 0, first = 0;
#pragma unroll
        for (int q = 0; q + 1 < TN_MAX; ++q) {
            const int e = g.end[q];
            j = l >= e ? q + 1 : j;
            first = l >= e ? e : first;
        }
        j = __builtin_amdgcn_readfirstlane(j);
        const GemmTnProb& p = g.p[j];
        t.M = p.M; t.N = p.N; t.A0 = p.A; t.B0 = p.B; t.C = p.C;
        tile_coords(l - first, (t.M + 255) / 256, (t.N + 255) / 256, bm, bn);
    }, smem);
}

// ---------------------------------------------------------------------------
// Grouped launch: up to GROUP_MAX independent products with 128x128 tiles, their contractions cut into parts when the
// tiles alone leave CUs idle.  For the products with a rank-r adapter matrix (an output of r columns or r rows with a long
// contraction: 2 to 32 tiles each) and for layers with few kept tokens: what they cost one by one is launches (5 us
// for the smallest kernel), blocks that wait for loads on a few CUs (a CU takes in about 60 B/ns whatever the number
// of active CUs), and a reduction each.  A launch has a fixed cost, though (scale * dY*b^T of 4096 rows, rank 64, K = 3072, six
// steps of 64 k in every block: 16 us and 6 us for the sum), so a single product of medium size gains nothing here.
// An item is one (tile, part); a part of a split tile leaves its fp32 accumulators in a 64 KB slot of its own and
// gemm_group_reduce_kernel adds the slots of a tile up in the order of the parts.  Blocks and reduction make the same plan
// from the live kept-token count, so the result is the same whether the count was known to the host or not.
// ---------------------------------------------------------------------------
struct GroupArgs {
    GemmGroupProb p[GROUP_MAX];
    int np;
    int n_cu;               // items that may be split over (and slots)
    const int32_t* n_dev;   // nullable: the live kept-token count (M in modes 0 and 2, K in mode 1), at most the one in p
    int gain;               // steps of 64 that parts have to take off the longest contraction
    float* slots;           // nullable: no splitting; n_cu slots and, behind them, the plan (one int)
    __host__ __device__ int32_t* plan() const { return reinterpret_cast<int32_t*>(slots + (size_t)n_cu * (128 * 128)); }
};

__host__ __device__ inline void group_sizes(const GemmGroupProb& p, int n_live, int& M, int& K) {
    M = p.mode != 1 && n_live < p.M ? n_live : p.M;
    K = p.mode == 1 && n_live < p.K ? n_live : p.K;
}
// Part sizes are numbered q = 2, 3, 4, 5, ...: 2, 3, 4, 6, 8, 12, ... steps of 64.
__host__ __device__ inline int group_step(int q) { return q & 1 ? 3 << ((q >> 1) - 1) : 1 << (q >> 1); }
// parts of a contraction of K, at least one
__host__ __device__ inline int group_parts(int K, int q) {
    const int k64 = (K + 63) >> 6, up = k64 + group_step(q) - 1;
    if (k64 <= 0) return 1;
    return q & 1 ? (up / 3) >> ((q >> 1) - 1) : up >> (q >> 1);
}
// Part size number of a launch: the smallest (at least 128 k: two steps) with which the items of all products fit one
// round of the CUs; -1, nothing is split, when even the whole tiles do not, or without slots.
static constexpr int GROUP_Q = 40;
// ... or when the longest contraction gets shorter by fewer than g.gain steps: a step is 0.35 to 0.5 us, against the launch that sums
// the parts up and their slots (GROUP_GAIN; GROUP_GAIN_ONE for a single product, whose sum is smaller).  Four products
// [4096, 64] of 48 and 16 steps, 128 tiles: 24 + 13 us in two parts, 33 whole; three of 48 steps, 96 tiles: 23 + 10 and 28; one, 32
// tiles: 16 + 6 in eight parts, 28 whole.  Contractions of up to 32 steps are faster whole whatever the rows (layer calls: H = 840, 215 rows 149
// and 172 us, H = 2048, 150 rows 167 and 172).  Those of 48 steps would be faster in four parts and more, which a batch of up to 1900 rows
// allows (H = 3072: 100 rows 202 and 210, 900 443 and 452, 1900 809 and 817), but with the count on the device their sums would have
// to be launched for longer batches too, where nothing is cut ([4096, 3072] 1216 and 1210, [4096 of 8192 in one sequence] 1436 and 1428).
__host__ __device__ inline int group_steps(const GroupArgs& g, int n_live) {        // of the longest contraction
    int most = 0;
#pragma unroll
    for (int j = 0; j < GROUP_MAX; ++j) {
        int M, K;
        group_sizes(g.p[j], n_live, M, K);
        const int k64 = (K + 63) >> 6;
        most = j < g.np && k64 > most ? k64 : most;
    }
    return most;
}
__host__ __device__ inline bool group_fits(const GroupArgs& g, int n_live, int q, bool& split) {
    int items = 0;
    split = false;
#pragma unroll
    for (int j = 0; j < GROUP_MAX; ++j) {
        int M, K;
        group_sizes(g.p[j], n_live, M, K);
        const int parts = group_parts(K, q);
        const bool used = j < g.np;
        items += used ? cdiv(M, 128) * cdiv(g.p[j].N, 128) * parts : 0;
        split |= used && parts > 1;
    }
    return items <= g.n_cu;
}
inline int group_plan_host(const GroupArgs& g, int n_live) {
    if (g.slots == nullptr) return -1;
    for (int q = 2; q < GROUP_Q; ++q) {
        bool split;
        const bool fits = group_fits(g, n_live, q, split);
        if (fits || !split) return split && group_steps(g, n_live) - group_step(q) >= g.gain ? q : -1;
    }
    return -1;
}
// The same with a candidate per lane: one after the other they cost every block several microseconds.
__device__ __forceinline__ int group_plan(const GroupArgs& g, int n_live) {
    if (g.slots == nullptr) return -1;
    const int q = 2 + (int)(threadIdx.x & 63);
    bool split = false;
    const bool fits = group_fits(g, n_live, q < GROUP_Q ? q : GROUP_Q - 1, split);
    const uint64_t done = __ballot(q < GROUP_Q && (fits || !split)), cut = __ballot(split);
    if (done == 0) return -1;
    const int first = __ffsll((unsigned long long)done) - 1;
    return ((cut >> first) & 1) && group_steps(g, n_live) - group_step(first + 2) >= g.gain ? first + 2 : -1;
}

// item -> product, tile and part; false past the last item
struct GroupItem {
    int j, M, K, m0, n0, parts, part;
};
__device__ __forceinline__ bool group_item(const GroupArgs& g, int n_live, int plan, int w, GroupItem& it) {
    it.j = -1;
    int tm_j = 1;
#pragma unroll
    for (int j = 0; j < GROUP_MAX; ++j) {
        int M, K;
        group_sizes(g.p[j], n_live, M, K);
        const int tm = cdiv(M, 128), parts = plan < 0 ? 1 : group_parts(K, plan);
        const int n = j < g.np ? tm * cdiv(g.p[j].N, 128) * parts : 0;
        if (it.j < 0 && w < n) { it.j = j; it.M = M; it.K = K; it.parts = parts; it.part = w; tm_j = tm; }
        w -= n;
    }
    if (it.j < 0) return false;
    const int t = it.part / it.parts;
    it.part -= t * it.parts;
    it.m0 = (t % tm_j) * 128;
    it.n0 = (t / tm_j) * 128;
    return true;
}

template <int MODE>
__device__ __forceinline__ void group_tile(const GroupArgs& ga, const GroupItem& it, int plan, int w, unsigned char* smem) {
    const GemmGroupProb& p = ga.p[it.j];
    GemmArgs g;
    g.A[0] = uniform_ptr(p.A); g.B[0] = uniform_ptr(p.B); g.K[0] = it.K; g.nseg = 1;
    g.C = uniform_ptr(p.C); g.M = it.M; g.N = p.N; g.beta = 0.f; g.alpha = p.alpha;
    g.n_dev = nullptr; g.a_idx = nullptr; g.a_rows = 0;
    const TileRef t{it.m0, it.n0, it.M, p.N, g.A[0], g.B[0], g.C};
    auto none = [](TileRef&) { return false; };
    if (it.parts > 1) {
        const int c = group_step(plan), pbeg = it.part * c, pend = min((it.K + 63) >> 6, pbeg + c);
        gemm_tiles<MODE, 2, 2, true, false>(g, it.K, t, none, smem, pbeg, pend, ga.slots + (int64_t)w * (128 * 128));
    } else {
        gemm_tiles<MODE, 2, 2, false, false>(g, it.K, t, none, smem);
    }
}

__global__ __launch_bounds__(256) void gemm_group_kernel(GroupArgs g) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int n_live = g.n_dev != nullptr ? __builtin_amdgcn_readfirstlane(max(*g.n_dev, 0)) : INT32_MAX;
    const int plan = __builtin_amdgcn_readfirstlane(group_plan(g, n_live));
    // for the reduction: made by every one of its blocks, the plan would cost it more than the sums (12 us for 4096 blocks)
    if (blockIdx.x == 0 && threadIdx.x == 0 && g.slots != nullptr) *g.plan() = plan;
    for (int w = blockIdx.x;; w += gridDim.x) {
        GroupItem it;
        if (!group_item(g, n_live, plan, w, it)) return;
        it.j = __builtin_amdgcn_readfirstlane(it.j);
        it.m0 = __builtin_amdgcn_readfirstlane(it.m0);
        it.n0 = __builtin_amdgcn_readfirstlane(it.n0);
        const int mode = g.p[it.j].mode;
        if (mode == 0) group_tile<0>(g, it, plan, w, smem);
        else if (mode == 1) group_tile<1>(g, it, plan, w, smem);
        else group_tile<2>(g, it, plan, w, smem);
        wait_vmcnt<0>();
        lds_barrier();          // the stages are free for the block's next item
    }
}

// C tile = alpha * (sum of its parts); tiles that were not split have been written already.  A block sums 8 rows of a
// tile, 4 columns per thread, eight parts in flight.  The grid has 16 blocks for every tile that the plan may hold.
__global__ __launch_bounds__(256) void gemm_group_reduce_kernel(GroupArgs g) {
    const int n_live = g.n_dev != nullptr ? max(*g.n_dev, 0) : INT32_MAX;
    const int plan = *g.plan();
    if (plan < 0) return;
    int t = (int)blockIdx.x >> 4, w0 = 0, jj = -1, Mj = 0, parts_j = 1, tm_j = 1, t_j = 0, w_j = 0;
#pragma unroll
    for (int j = 0; j < GROUP_MAX; ++j) {
        int M, K;
        group_sizes(g.p[j], n_live, M, K);
        const int tm = cdiv(M, 128), tiles = j < g.np ? tm * cdiv(g.p[j].N, 128) : 0;
        const int parts = group_parts(K, plan);
        if (jj < 0 && t < tiles) { jj = j; Mj = M; parts_j = parts; tm_j = tm; t_j = t; w_j = w0; }
        t -= tiles;
        w0 += tiles * parts;
    }
    if (jj < 0 || parts_j == 1) return;
    const GemmGroupProb& p = g.p[jj];
    const int row = ((int)blockIdx.x & 15) * 8 + ((int)threadIdx.x >> 5), col = ((int)threadIdx.x & 31) * 4;
    const int m = (t_j % tm_j) * 128 + row, n = (t_j / tm_j) * 128 + col;
    if (m >= Mj || n >= p.N) return;            // N is a multiple of 8
    const float* src = g.slots + (int64_t)(w_j + t_j * parts_j) * (128 * 128) + row * 128 + col;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int k = 0; k < parts_j; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(src + (int64_t)k * (128 * 128));
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    uint2 o;
    o.x = pack_bf16x2(p.alpha * s.x, p.alpha * s.y);
    o.y = pack_bf16x2(p.alpha * s.z, p.alpha * s.w);
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.C) + (int64_t)m * p.N + n) = o;
}

// ---------------------------------------------------------------------------
// fp32 check-mode GEMM: 64x64 tile, 16-wide K step, 4x4 outputs per thread
// ---------------------------------------------------------------------------
template <int MODE>
__global__ __launch_bounds__(256) void gemm_f32_kernel(GemmArgs g) {
    __shared__ float As[16][64 + 4];
    __shared__ float Bs[16][64 + 4];
    const int tid = threadIdx.x;
    const int tiles_m = (g.M + 63) / 64;        // of the upper bound: the grid was sized for it
    const int m0 = (blockIdx.x % tiles_m) * 64, n0 = (blockIdx.x / tiles_m) * 64;
    if (g.n_dev != nullptr) {
        const int n = live_rows(MODE != 1 ? g.M : g.K[0], g.n_dev);
        if (MODE != 1) g.M = n;
        else g.K[0] = n;
        if (m0 >= g.M) return;
    }
    const int tx = tid & 15, ty = tid >> 4;
    float acc[4][4] = {};
    for (int s = 0; s < g.nseg; ++s) {
        const float* A = static_cast<const float*>(g.A[s]);
        const float* B = static_cast<const float*>(g.B[s]);
        const int K = g.K[s];
        for (int k0 = 0; k0 < K; k0 += 16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = tid + 256 * i;      // 0..1023
                int kk, r;
                if (MODE != 1) { kk = e & 15; r = e >> 4; } else { r = e & 63; kk = e >> 6; }
                const bool ka = k0 + kk < K;
                float av = 0.f, bv = 0.f;
                if (ka && m0 + r < g.M) {
                    const int64_t arow = (MODE == 0 && s == 0 && g.a_idx != nullptr) ? g.a_idx[m0 + r] : m0 + r;
                    av = MODE != 1 ? A[arow * K + k0 + kk] : A[(int64_t)(k0 + kk) * g.M + m0 + r];
                }
                if (ka && n0 + r < g.N)
                    bv = MODE == 0 ? B[(int64_t)(n0 + r) * K + k0 + kk] : B[(int64_t)(k0 + kk) * g.N + n0 + r];
                As[kk][r] = av;
                Bs[kk][r] = bv;
            }
            __syncthreads();
#pragma unroll
            for (int kk = 0; kk < 16; ++kk) {
                float a[4], b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) { a[i] = As[kk][ty * 4 + i]; b[i] = Bs[kk][tx * 4 + i]; }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] += a[i] * b[j];
            }
            __syncthreads();
        }
    }
    float* C = static_cast<float*>(g.C);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + ty * 4 + i;
        if (m >= g.M) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = n0 + tx * 4 + j;
            if (n >= g.N) continue;
            float* p = C + (int64_t)m * g.N + n;
            *p = (g.beta != 0.f) ? g.alpha * acc[i][j] + g.beta * *p : g.alpha * acc[i][j];
        }
    }
}


// per-lane load and store offsets are 32-bit with the upper half reserved for "out of range"
static bool offsets_fit(int64_t M, int64_t N, int64_t K) {
    const int64_t lim = (int64_t)1 << 31;
    return M * K * 2 < lim && N * K * 2 < lim && (M + 256) * N * 2 < lim;
}

// C = the sum of the parts of a product that was cut into some
__global__ __launch_bounds__(256) void gemm_nt_sum_kernel(NtParts pt, int M, bf16_t* __restrict__ C) {
    int per;
    const int parts = pt.count(M, per), vpr = pt.N / 8;
    const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (v >= (int64_t)M * vpr) return;
    const int j = (int)(v / vpr), c = (int)(v % vpr) * 8;
    float o[8];
    pt.load(M, parts, j, c, o);
    Vec<bf16_t>::store(C + (int64_t)j * pt.N + c, o);
}

hipError_t launch_gemm_nt_sum(const NtParts& parts, int M, void* C, hipStream_t st) {
    int per;
    if (M <= 0 || parts.count(M, per) == 1) return hipSuccess;
    gemm_nt_sum_kernel<<<ceil_div((int64_t)M * parts.N, 256 * 8), 256, 0, st>>>(parts, M, (bf16_t*)C);
    return hipGetLastError();
}

NtParts gemm_nt_parts(int dtype, const GemmSeg* segs, int nseg, int N, float* slots) {
    NtParts p{slots, N, 0, compute_units(), 0};
    if (dtype != CF_BF16 || slots == nullptr) return p;
    for (int s = 0; s < nseg; ++s) p.pairs += ceil_div(segs[s].K, 64);
    // the more tiles, the fewer parts: the last number of tile rows with more than one
    const int tn = ceil_div(N, 128);
    int per;
    for (int tm = 1; 2 * tm * tn <= p.n_cu; ++tm) {
        p.max_rows = tm * 128;
        if (p.count(tm * 128, per) == 1) {
            p.max_rows = (tm - 1) * 128;
            break;
        }
    }
    return p;
}

hipError_t launch_gemm_nt(int dtype, const GemmSeg* segs, int nseg, void* C, int M, int N, hipStream_t st, const int32_t* n_dev,
                          const int32_t* a_idx, int64_t a_rows, const NtParts* parts) {
    if (M <= 0 || N <= 0) return hipSuccess;
    if (a_idx != nullptr && a_rows <= 0) return hipErrorInvalidValue;
    if (nseg > MAX_SEG) return hipErrorInvalidValue;
    GemmArgs g{};
    for (int s = 0; s < nseg; ++s) {
        if (segs[s].K <= 0) return hipErrorInvalidValue;
        g.A[s] = segs[s].A;
        g.B[s] = segs[s].B;
        g.K[s] = segs[s].K;
        if (dtype == CF_BF16 && !offsets_fit(M, N, segs[s].K)) return hipErrorInvalidValue;
    }
    g.nseg = nseg;
    g.C = C; g.M = M; g.N = N; g.alpha = 1.f; g.sub = 1; g.tile_n = 256;
    g.n_dev = n_dev; g.a_idx = a_idx; g.a_rows = a_rows;
    if (dtype == CF_F32) {
        gemm_f32_kernel<0><<<ceil_div(M, 64) * ceil_div(N, 64), 256, 0, st>>>(g);
        return hipGetLastError();
    }
    if (a_idx != nullptr && a_rows * g.K[0] * 2 >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    static std::atomic<uint64_t> lds_ok{0};
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&gemm_nt_kernel), GEMM_SMEM, lds_ok);
    if (e != hipSuccess) return e;
    if (parts != nullptr) g.parts = *parts;
    int per, items = plan_launch(M, N, compute_units(), g.n_full, g.sub, g.tile_n);
    const int np = g.parts.count(M, per);
    if (np > 1) items = ceil_div(M, 128) * ceil_div(N, 128) * np;
    // a block walks through its items; with a device-side count the blocks plan for themselves (for
    // as many blocks as CUs) and those without an item leave at once
    const int grid = n_dev != nullptr ? compute_units() : std::min(items, compute_units());
    gemm_nt_kernel<<<grid, 256, GEMM_SMEM, st>>>(g);
    return hipGetLastError();
}

hipError_t launch_gemm_tn(int dtype, const GemmTnProb* probs, int np, int K, float beta, hipStream_t st, bool c_f32,
                          const int32_t* n_dev, const GainGrads* gains) {
    if (np < 1 || np > TN_MAX) return hipErrorInvalidValue;
    if (c_f32 && dtype == CF_BF16 && beta != 1.f) return hipErrorInvalidValue;
    if (gains != nullptr && (K <= 0 || dtype == CF_F32)) {
        const hipError_t e = launch_gain_grads(dtype, *gains, c_f32, st);
        if (e != hipSuccess) return e;
    }
    if (K <= 0) {           // empty contraction: C = beta*C; only beta in {0,1} is supported by the API
        for (int j = 0; j < np && beta == 0.f; ++j) {
            const hipError_t e = launch_fill_zero(probs[j].C, (size_t)probs[j].M * probs[j].N * dtype_size(dtype), st);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    TnArgs g{};
    g.K[0] = K; g.nseg = 1; g.beta = beta; g.alpha = 1.f; g.n_dev = n_dev;
    if (dtype == CF_F32) {
        for (int j = 0; j < np; ++j) {
            g.A[0] = probs[j].A; g.B[0] = probs[j].B; g.C = probs[j].C; g.M = probs[j].M; g.N = probs[j].N;
            gemm_f32_kernel<1><<<ceil_div(g.M, 64) * ceil_div(g.N, 64), 256, 0, st>>>(g);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    int tiles = 0;
    for (int j = 0; j < TN_MAX; ++j) {
        if (j < np) {
            const GemmTnProb& p = probs[j];
            if (p.M <= 0 || p.N <= 0 || !offsets_fit(p.M, p.N, K)) return hipErrorInvalidValue;
            g.p[j] = p;
            tiles += ceil_div(p.M, 256) * ceil_div(p.N, 256);
        }
        g.end[j] = tiles;       // behind the last product: no tile there
    }
    static std::atomic<uint64_t> lds_ok{0}, lds_ok_f32{0};
    void (*const kernel)(TnArgs) = c_f32 ? gemm_tn_kernel<true> : gemm_tn_kernel<false>;
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), GEMM_SMEM, c_f32 ? lds_ok_f32 : lds_ok);
    if (e != hipSuccess) return e;
    plan_tiles(tiles, compute_units(), g.n_full, g.sub);
    g.n_blocks = std::min(g.n_full + (tiles - g.n_full) * g.sub, compute_units());
    int more = 0;
    if (gains != nullptr && tiles > compute_units()) {
        g.gain = *gains;
        more = gain_grad_units(gains->H);
    } else if (gains != nullptr) {
        // Up to one round a launch of their own, as the number of launches of such a call has always been, which test_gpu_routes.py
        // holds to.  Not for speed: beside the products 94 layer calls of 7 to 228 tiles are 1.03 times as fast (1.01 to 1.07, 1 to 7 us).
        const hipError_t eg = launch_gain_grads(dtype, *gains, c_f32, st);
        if (eg != hipSuccess) return eg;
    }
    kernel<<<g.n_blocks + more, 256, GEMM_SMEM, st>>>(g);
    return hipGetLastError();
}

size_t gemm_group_slot_bytes() { return (size_t)compute_units() * 128 * 128 * sizeof(float) + 256; }

hipError_t launch_gemm_group(int dtype, const GemmGroupProb* probs, int np, hipStream_t st, float* slots,
                             const int32_t* n_dev) {
    if (np < 1 || np > GROUP_MAX) return hipErrorInvalidValue;
    if (dtype == CF_F32) {
        for (int j = 0; j < np; ++j) {
            const GemmGroupProb& p = probs[j];
            GemmArgs g{};
            g.A[0] = p.A; g.B[0] = p.B; g.K[0] = p.K; g.nseg = 1; g.C = p.C; g.M = p.M; g.N = p.N; g.alpha = p.alpha;
            g.n_dev = n_dev;
            const int grid = ceil_div(p.M, 64) * ceil_div(p.N, 64);
            if (p.mode == 0) gemm_f32_kernel<0><<<grid, 256, 0, st>>>(g);
            else if (p.mode == 1) gemm_f32_kernel<1><<<grid, 256, 0, st>>>(g);
            else gemm_f32_kernel<2><<<grid, 256, 0, st>>>(g);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    GroupArgs g{};
    int64_t tiles = 0;
    bool all_tn = true;
    for (int j = 0; j < np; ++j) {
        const GemmGroupProb& p = probs[j];
        if (p.M <= 0 || p.N <= 0 || p.K <= 0) return hipErrorInvalidValue;
        if (!offsets_fit(p.M, p.N, p.K)) return hipErrorInvalidValue;
        g.p[j] = p;
        tiles += (int64_t)ceil_div(p.M, 128) * ceil_div(p.N, 128);
        all_tn = all_tn && p.mode == 1;
    }
    g.np = np; g.n_cu = compute_units(); g.n_dev = n_dev; g.slots = slots; g.gain = np == 1 ? GROUP_GAIN_ONE : GROUP_GAIN;
    // no live count can lead to parts: their sum is not launched (products over the kept tokens have the same tiles whatever the count, and
    // are cut alike)
    if (group_steps(g, INT32_MAX) - group_step(2) < g.gain || (all_tn && 2 * tiles > g.n_cu)) g.slots = slots = nullptr;
    static std::atomic<uint64_t> lds_ok{0};
    hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&gemm_group_kernel), GEMM_SMEM, lds_ok);
    if (e != hipSuccess) return e;
    // a live count below the bound may be split although the bound is not: the launches are sized for either
    const bool may_split = slots != nullptr && (n_dev != nullptr || group_plan_host(g, INT32_MAX) >= 0);
    const int grid = (int)(may_split ? g.n_cu : std::min<int64_t>(tiles, g.n_cu));
    gemm_group_kernel<<<grid, 256, GEMM_SMEM, st>>>(g);
    e = hipGetLastError();
    if (e != hipSuccess || !may_split) return e;
    // a plan with parts has at most n_cu items, so at most n_cu / 2 of its tiles are split; whole ones count too
    const int rtiles = (int)std::min<int64_t>(tiles, g.n_cu);
    gemm_group_reduce_kernel<<<16 * rtiles, 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace cf
