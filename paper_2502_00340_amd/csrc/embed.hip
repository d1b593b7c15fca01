// Token embeddings and their gradient.  y_t = s * E[tok_t] is a gather: HBM-bound, rows in and rows out.  The gradient dE[c] (+)= s * sum of the dx rows
// whose token is c is a sum over equal tokens: the rows are put in the order (token, row), so that a token's rows stand together and are added
// up in ascending order, whatever the launch does.  It reads the rows once and touches, in a main gradient, no other row of the table.
#include "common.h"
#include "mfma_util.h"

namespace cf {

// ---- forward -------------------------------------------------------------------------------------------------
// 8192 rows of [128256, 4096] bf16: 17.6 us, 5.6 TB/s; a copy of as much in one piece reaches 6.3.

template <typename T>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const T* __restrict__ table, const int64_t* __restrict__ tokens, int64_t n, int V, int vpr,
                                                        int lanes, int rpb, float scale, T* __restrict__ y) {
    constexpr int VN = Vec<T>::N;
    const int r = threadIdx.x / lanes, c0 = threadIdx.x % lanes;
    if (r >= rpb) return;
    for (int64_t j = (int64_t)blockIdx.x * rpb + r; j < n; j += (int64_t)gridDim.x * rpb) {
        const int64_t t = tokens[j];
        const bool live = t >= 0 && t < V;
        const T* src = table + (live ? t : 0) * vpr * VN;
        T* dst = y + j * vpr * VN;
        for (int c = c0; c < vpr; c += lanes) {
            u32x4_t w = {0u, 0u, 0u, 0u};
            if (live) {
                w = *reinterpret_cast<const u32x4_t*>(src + c * VN);
                if (scale != 1.f) {
                    float o[VN];
                    Vec<T>::load(src + c * VN, o);
#pragma unroll
                    for (int e = 0; e < VN; ++e) o[e] *= scale;
                    Vec<T>::store(dst + c * VN, o);
                    continue;
                }
            }
            *reinterpret_cast<u32x4_t*>(dst + c * VN) = w;
        }
    }
}

template <typename T>
static void launch_embed_fwd(const void* table, const int64_t* tokens, int64_t n, int V, int H, float scale, void* y, hipStream_t st) {
    const int vpr = H / Vec<T>::N;
    int lanes = 256;
    while (lanes > 1 && lanes / 2 >= vpr) lanes /= 2;
    const int rpb = 256 / lanes;
    const int64_t blocks = (n + rpb - 1) / rpb;
    embed_fwd_kernel<T><<<(int)(blocks < MAX_GRID ? blocks : MAX_GRID), 256, 0, st>>>((const T*)table, tokens, n, V, vpr, lanes, rpb, scale, (T*)y);
}

// ---- the rows in the order (token, row) ----------------------------------------------------------------------
// A block sorts a span of up to 8192 rows in LDS: passes of nine bits, lowest first, each keeping the order of what is equal.  A wave takes a
// contiguous part of the span, 64 rows at a time; rows of one wave and round that share a digit find each other by nine ballots.  Two passes do for
// 2^18 tokens (4096 rows in one block: 16.8 us).  Spans are merged by rank: a row's place is its place in its span and, for each other span, the number of rows there that go ahead of it.

constexpr int SPAN = 8192, DIGIT_BITS = 9, DIGITS = 1 << DIGIT_BITS, SORT_WAVES = 16, SORT_THREADS = 64 * SORT_WAVES, PER_THREAD = SPAN / SORT_THREADS;
constexpr int SORT_LDS = SPAN * 4 + SPAN * 2 + SORT_WAVES * DIGITS * 2 + 64;

struct SortArgs {
    const int64_t* tokens;
    const int32_t *idx, *n_dev;
    int n_max, V, passes;
    int32_t *tok, *row;     // out: sorted, span by span
    int spans;
    u32x4_t* zero;          // nullable: the blocks behind those of the spans clear zero[0 .. n_zero)
    int64_t n_zero;
};

// block of blocks, of `threads`; as a rule a vector a thread.  Past the caches: 8 tables of 169 MB in turn 37.8 us a call, through them 40.6 (a call that is waited for takes
// 57 and 51); most of them cleared beside the sums instead, where the ordered tokens tell which rows nobody adds to, 39.7.
__device__ __forceinline__ void clear_table(const SortArgs& a, int block, int blocks, int threads) {
    const int64_t stride = (int64_t)blocks * threads;
    for (int64_t i = (int64_t)block * threads + threadIdx.x; i < a.n_zero; i += stride) __builtin_nontemporal_store(u32x4_t{0u, 0u, 0u, 0u}, a.zero + i);
}

__global__ __launch_bounds__(SORT_THREADS) void embed_sort_kernel(SortArgs a) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if ((int)blockIdx.x >= a.spans) {
        clear_table(a, (int)blockIdx.x - a.spans, (int)gridDim.x - a.spans, SORT_THREADS);
        return;
    }
    extern __shared__ __align__(16) unsigned char smem[];
    unsigned* skey = reinterpret_cast<unsigned*>(smem);
    uint16_t* sval = reinterpret_cast<uint16_t*>(smem + SPAN * 4);
    uint16_t* cnt = sval + SPAN;                        // [wave][digit]
    int* tot = reinterpret_cast<int*>(cnt + SORT_WAVES * DIGITS);
    const int n_rows = live_rows(a.n_max, a.n_dev), first = (int)blockIdx.x * SPAN, m = min(n_rows - first, SPAN);
    if (m <= 0) return;
    const int rounds = (m + SORT_THREADS - 1) / SORT_THREADS;          // of 64 rows, for each wave
    const int at0 = wave * rounds * 64 + lane;
    unsigned key[PER_THREAD];
    int val[PER_THREAD];
#pragma unroll
    for (int r = 0; r < PER_THREAD; ++r) {
        const int i = at0 + r * 64;
        key[r] = 0;
        val[r] = i;
        if (r < rounds && i < m) {
            const int j = first + i;
            const int64_t t = a.tokens[a.idx != nullptr ? a.idx[j] : j];
            key[r] = t >= 0 && t < a.V ? (unsigned)t : (unsigned)a.V;      // what is no token goes last
        }
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * DIGIT_BITS;
        for (int i = tid; i < SORT_WAVES * DIGITS / 2; i += SORT_THREADS) reinterpret_cast<unsigned*>(cnt)[i] = 0u;
        __syncthreads();
        volatile uint16_t* mine = cnt + wave * DIGITS;
        int rank[PER_THREAD];
#pragma unroll
        for (int r = 0; r < PER_THREAD; ++r) {
            rank[r] = 0;
            if (r < rounds) {                           // the same for all threads
                const bool valid = at0 + r * 64 < m;
                const unsigned d = (key[r] >> shift) & (DIGITS - 1);
                uint64_t same = __ballot(valid);
#pragma unroll
                for (int b = 0; b < DIGIT_BITS; ++b) {
                    const uint64_t bal = __ballot((d >> b) & 1u);
                    same &= (d >> b) & 1u ? bal : ~bal;
                }
                if (valid) {
                    const int before = mine[d];         // read by all, then written by the first lane: a wave's LDS accesses keep their order
                    const int below = __popcll(same & ((1ull << lane) - 1ull));
                    rank[r] = before + below;
                    __builtin_amdgcn_wave_barrier();
                    if (below == 0) mine[d] = (uint16_t)(before + __popcll(same));
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
        __syncthreads();
        // a digit's rows of wave w start behind all rows of smaller digits and those of the waves ahead of it
        int total = 0;
        if (tid < DIGITS) {
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) {
                const int c = cnt[w * DIGITS + tid];
                cnt[w * DIGITS + tid] = (uint16_t)total;
                total += c;
            }
        }
        int incl = total;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(incl, o, 64);
            if (lane >= o) incl += v;
        }
        if (tid < DIGITS && lane == 63) tot[wave] = incl;
        __syncthreads();
        if (tid < DIGITS) {
            int base = incl - total;
#pragma unroll
            for (int w = 0; w < DIGITS / 64; ++w) base += w < wave ? tot[w] : 0;
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) cnt[w * DIGITS + tid] = (uint16_t)(cnt[w * DIGITS + tid] + base);
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < PER_THREAD; ++r) {
            if (r < rounds && at0 + r * 64 < m) {
                const int to = cnt[wave * DIGITS + ((key[r] >> shift) & (DIGITS - 1))] + rank[r];
                skey[to] = key[r];
                sval[to] = (uint16_t)val[r];
            }
        }
        __syncthreads();
        if (pass + 1 == a.passes) break;
#pragma unroll
        for (int r = 0; r < PER_THREAD; ++r) {
            if (r < rounds && at0 + r * 64 < m) {
                key[r] = skey[at0 + r * 64];
                val[r] = sval[at0 + r * 64];
            }
        }
    }
    for (int i = tid; i < m; i += SORT_THREADS) {
        a.tok[first + i] = (int32_t)skey[i];
        a.row[first + i] = first + (int)sval[i];
    }
}

// Up to a span the rows are put in order by counting instead, on all CUs in one launch: a row's place is the number of rows with a smaller token and of rows
// ahead of it with the same one.  n^2 comparisons of keys in LDS; a wave takes a row.  4096 rows 6.0 us, of
// which the keys' loads through the index are half; with 16 lanes a row in blocks of 256 threads 10.9.
constexpr int RANK_ROWS = 16, RANK_THREADS = 64 * RANK_ROWS;

__global__ __launch_bounds__(RANK_THREADS) void embed_rank_kernel(SortArgs a, int rank_blocks) {
    __shared__ __align__(16) int key[SPAN];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= rank_blocks) {
        clear_table(a, (int)blockIdx.x - rank_blocks, (int)gridDim.x - rank_blocks, RANK_THREADS);
        return;
    }
    const int n_rows = live_rows(a.n_max, a.n_dev), j0 = blockIdx.x * RANK_ROWS;
    if (j0 >= n_rows) return;
    const int padded = (n_rows + 255) & ~255;           // keys of rows that do not exist are larger than every token
    constexpr int U = 4;
    for (int i0 = tid; i0 < padded; i0 += U * RANK_THREADS) {
        int at[U];
        int64_t t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = min(i0 + u * RANK_THREADS, n_rows - 1);
            at[u] = a.idx != nullptr ? a.idx[i] : i;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) t[u] = a.tokens[at[u]];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * RANK_THREADS;
            if (i < padded) key[i] = i >= n_rows ? INT32_MAX : t[u] >= 0 && t[u] < a.V ? (int)t[u] : a.V;
        }
    }
    __syncthreads();
    const int j = __builtin_amdgcn_readfirstlane(j0 + (tid >> 6)), lane = tid & 63;
    if (j >= n_rows) return;
    const int k = key[j], border = j & ~255;            // keys ahead of row j count up to k, those behind it below k
    int rank = 0;
    auto count = [&](int from, int to, int below) __attribute__((always_inline)) {
#pragma unroll 4
        for (int i = from + lane * 4; i < to; i += 256) {
            const int4 v = *reinterpret_cast<const int4*>(&key[i]);
            rank += (v.x < below) + (v.y < below) + (v.z < below) + (v.w < below);
        }
    };
    count(0, border, k + 1);
    count(border + 256, padded, k);
    const int i = border + lane * 4;
    const int4 v = *reinterpret_cast<const int4*>(&key[i]);
    rank += (v.x < k + (i < j)) + (v.y < k + (i + 1 < j)) + (v.z < k + (i + 2 < j)) + (v.w < k + (i + 3 < j));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) rank += __shfl_xor(rank, o, 64);
    if (lane == 0) {
        a.tok[rank] = k;
        a.row[rank] = j;
    }
}

// rows of s[0 .. m) with a token below t, or up to it
__device__ __forceinline__ int rank_in(const int32_t* __restrict__ s, int m, int t, bool equal_too) {
    int lo = 0, hi = m;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const bool ahead = equal_too ? s[mid] <= t : s[mid] < t;
        lo = ahead ? mid + 1 : lo;
        hi = ahead ? hi : mid;
    }
    return lo;
}

__global__ __launch_bounds__(256) void embed_merge_kernel(const int32_t* __restrict__ tok, const int32_t* __restrict__ row, int n_max,
                                                          const int32_t* __restrict__ n_dev, int32_t* __restrict__ tok_out,
                                                          int32_t* __restrict__ row_out) {
    const int n_rows = live_rows(n_max, n_dev);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n_rows; i += (int64_t)gridDim.x * 256) {
        const int span = (int)(i / SPAN), t = tok[i];
        int64_t to = i % SPAN;
        for (int s = 0; (int64_t)s * SPAN < n_rows; ++s)
            if (s != span) to += rank_in(tok + (int64_t)s * SPAN, min(SPAN, n_rows - s * SPAN), t, s < span);
        tok_out[to] = t;
        row_out[to] = row[i];
    }
}

// ---- sums ----------------------------------------------------------------------------------------------------
// A block takes CH rows of that order, and TILE columns.  All its loads are asked for at once (rows, and the main gradient's old values); then the
// rows are added up one by one, and a token's sum leaves where its last row has been added.  A token whose rows reach over the border of a block leaves parts: [chunk][0]
// of one that began ahead of the chunk, [chunk][1] of one that begins here and goes on.  embed_join_kernel adds these up in order.
// 4096 rows of 4096 bf16, log-uniform tokens, into an fp32 table: 110 MB in 21 us, 5.2 TB/s.
constexpr int CH = 8;

struct SumArgs {
    const int32_t *tok, *row, *n_dev;
    int n_max, V, H;
    const void* dx;
    float scale;
    void* out;
    float* part;
};

template <typename T, bool MAIN>
__device__ __forceinline__ void embed_out(const SumArgs& a, int t, int c, const float (&s)[Vec<T>::N], const float (&old)[Vec<T>::N]) {
    constexpr int VN = Vec<T>::N;
    float o[VN];
#pragma unroll
    for (int e = 0; e < VN; ++e) o[e] = MAIN ? fmaf(a.scale, s[e], old[e]) : a.scale * s[e];
    if constexpr (MAIN) {
        float* p = (float*)a.out + (int64_t)t * a.H + c;
#pragma unroll
        for (int q = 0; q < VN / 4; ++q) reinterpret_cast<float4*>(p)[q] = make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
    } else {
        Vec<T>::store((T*)a.out + (int64_t)t * a.H + c, o);
    }
}

template <typename T, int NT, bool MAIN>
__global__ __launch_bounds__(NT) void embed_sum_kernel(SumArgs a) {
    constexpr int VN = Vec<T>::N;
    const int n_rows = live_rows(a.n_max, a.n_dev), vpr = a.H / VN, tiles = (vpr + NT - 1) / NT;
    const int64_t units = (int64_t)((n_rows + CH - 1) / CH) * tiles;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int chunk = (int)(u / tiles), p0 = chunk * CH, v = (int)(u % tiles) * NT + threadIdx.x;
        int t[CH + 2];              // tokens of rows p0 - 1 .. p0 + CH; V: none
#pragma unroll
        for (int i = 0; i < CH + 2; ++i) {
            const int p = p0 + i - 1;
            t[i] = p >= 0 && p < n_rows ? a.tok[p] : a.V;
        }
        if (t[1] >= a.V) break;     // what is no token stands last
        const bool mine = v < vpr;
        const int c = (mine ? v : 0) * VN;
        u32x4_t x[CH];
        float old[CH][MAIN ? VN : 1];
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (t[i + 1] < a.V) x[i] = *reinterpret_cast<const u32x4_t*>((const T*)a.dx + (int64_t)a.row[p0 + i] * a.H + c);
        if constexpr (MAIN) {
            bool whole = t[0] != t[1];          // the token of row i began in this chunk
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const bool ends = t[i + 2] != t[i + 1];
                if (whole && ends && t[i + 1] < a.V) {
                    const float4* p = reinterpret_cast<const float4*>((const float*)a.out + (int64_t)t[i + 1] * a.H + c);
#pragma unroll
                    for (int q = 0; q < VN / 4; ++q) {
                        const float4 w = p[q];
                        old[i][4 * q] = w.x; old[i][4 * q + 1] = w.y; old[i][4 * q + 2] = w.z; old[i][4 * q + 3] = w.w;
                    }
                }
                whole |= ends;
            }
        }
        if (!mine) continue;
        float s[VN];
#pragma unroll
        for (int e = 0; e < VN; ++e) s[e] = 0.f;
        bool whole = t[0] != t[1];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (t[i + 1] >= a.V) break;
            const bool ends = t[i + 2] != t[i + 1];
            float o[VN];
            Vec<T>::load(reinterpret_cast<const T*>(&x[i]), o);
#pragma unroll
            for (int e = 0; e < VN; ++e) s[e] += o[e];
            if (ends || i == CH - 1) {
                if (whole && ends) {
                    if constexpr (MAIN) embed_out<T, true>(a, t[i + 1], c, s, old[i]);
                    else embed_out<T, false>(a, t[i + 1], c, s, s);
                } else {
                    float* p = a.part + ((int64_t)chunk * 2 + (whole ? 1 : 0)) * a.H + c;
#pragma unroll
                    for (int q = 0; q < VN / 4; ++q)
                        reinterpret_cast<float4*>(p)[q] = make_float4(s[4 * q], s[4 * q + 1], s[4 * q + 2], s[4 * q + 3]);
                }
#pragma unroll
                for (int e = 0; e < VN; ++e) s[e] = 0.f;
                whole = true;
            }
        }
    }
}

// The tokens whose rows reach over chunks.  A wave takes a chunk and 256 columns; it has work where a token begins in the chunk that goes on in the next one.
// Parts are added in order, 16 of them in flight.  Those rows, log-uniform tokens: 6.1 us, latency; blocks of 16 waves that share a token 14.6.  A long run is one wave's
// work: whole calls for 8192 rows of 840 with uniform tokens, half of one token and all of one token 28, 51 and 75 us, of 65536 rows of 2048 299, 505 and 565.
template <typename T, bool MAIN>
__global__ __launch_bounds__(256) void embed_join_kernel(SumArgs a) {
    const int n_rows = live_rows(a.n_max, a.n_dev), chunks = (n_rows + CH - 1) / CH, tiles = (a.H + 255) / 256, lane = threadIdx.x & 63;
    const int64_t items = (int64_t)(chunks - 1) * tiles, stride = (int64_t)gridDim.x * 4;          // nothing goes on behind the last chunk
    for (int64_t it = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); it < items; it += stride) {
        const int chunk = (int)(it / tiles), p1 = chunk * CH + CH, c = (int)(it % tiles) * 256 + lane * 4;
        // one load for what tells whether there is work, and, with the first 64 chunks behind this one, how much
        const int t = a.tok[p1 - 1], before = a.tok[chunk > 0 ? p1 - CH - 1 : 0];
        const int k0 = chunk + 1 + lane, ahead = a.tok[(k0 < chunks ? k0 : chunk + 1) * CH];
        if (t >= a.V || (chunk > 0 && before == t)) continue;
        uint64_t same = __ballot(k0 < chunks && ahead == t);
        if ((same & 1) == 0) continue;
        int parts = 1 + __popcll(same);                            // this chunk's and those of the chunks that begin with the token
        for (int k = chunk + 65; same == ~0ull; k += 64) {
            same = __ballot(k + lane < chunks && a.tok[(k + lane < chunks ? k + lane : 0) * CH] == t);
            parts += __popcll(same);
        }
        if (c >= a.H) continue;
        const int64_t at = (int64_t)t * a.H + c;
        float4 old = make_float4(0.f, 0.f, 0.f, 0.f);
        if constexpr (MAIN) old = *reinterpret_cast<const float4*>((const float*)a.out + at);
        const float* p = a.part + (int64_t)chunk * 2 * a.H + c;
        float4 s = *reinterpret_cast<const float4*>(p + a.H);
        for (int k = 1; k < parts; k += 16) {
            float4 w[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) w[u] = *reinterpret_cast<const float4*>(p + (int64_t)min(k + u, parts - 1) * 2 * a.H);
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                const bool have = k + u < parts;
                s.x += have ? w[u].x : 0.f; s.y += have ? w[u].y : 0.f; s.z += have ? w[u].z : 0.f; s.w += have ? w[u].w : 0.f;
            }
        }
        if constexpr (MAIN) {
            *reinterpret_cast<float4*>((float*)a.out + at) =
                make_float4(fmaf(a.scale, s.x, old.x), fmaf(a.scale, s.y, old.y), fmaf(a.scale, s.z, old.z), fmaf(a.scale, s.w, old.w));
        } else {
            T* o = (T*)a.out + at;
            o[0] = narrow_one<T>(a.scale * s.x); o[1] = narrow_one<T>(a.scale * s.y);
            o[2] = narrow_one<T>(a.scale * s.z); o[3] = narrow_one<T>(a.scale * s.w);
        }
    }
}

// ---- few rows ------------------------------------------------------------------------------------------------
// One launch instead of three: each row's block finds the rows with its token among up to 256, leaves if one of them is ahead, and adds them up in order.
constexpr int FEW_ROWS = 256;

template <typename T, bool MAIN>
__global__ __launch_bounds__(256) void embed_few_kernel(SumArgs a, const int64_t* __restrict__ tokens, const int32_t* __restrict__ idx) {
    constexpr int VN = Vec<T>::N, U = 8;
    __shared__ int key[FEW_ROWS], list[FEW_ROWS];
    __shared__ uint64_t same[4];
    const int n_rows = live_rows(a.n_max, a.n_dev), tid = threadIdx.x, wave = tid >> 6, vpr = a.H / VN, tiles = (vpr + 255) / 256, j = (int)blockIdx.x / tiles;
    if (j >= n_rows) return;
    int mine = a.V;
    if (tid < n_rows) {
        const int64_t t = tokens[idx != nullptr ? idx[tid] : tid];
        if (t >= 0 && t < a.V) mine = (int)t;
    }
    key[tid] = mine;
    __syncthreads();
    const int t = key[j];
    const bool hit = mine == t;
    const uint64_t b = __ballot(hit);
    if ((tid & 63) == 0) same[wave] = b;
    __syncthreads();
    if (t >= a.V) return;
    int at = __popcll(b & ((1ull << (tid & 63)) - 1ull)), n = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int c = __popcll(same[w]);
        at += w < wave ? c : 0;
        n += c;
    }
    if (hit) list[at] = tid;
    __syncthreads();
    if (list[0] != j) return;
    const int v = (int)blockIdx.x % tiles * 256 + tid;
    if (v >= vpr) return;
    const int c = v * VN;
    float old[VN] = {}, s[VN] = {};
    if constexpr (MAIN) {
        const float4* p = reinterpret_cast<const float4*>((const float*)a.out + (int64_t)t * a.H + c);
#pragma unroll
        for (int q = 0; q < VN / 4; ++q) {
            const float4 w = p[q];
            old[4 * q] = w.x; old[4 * q + 1] = w.y; old[4 * q + 2] = w.z; old[4 * q + 3] = w.w;
        }
    }
    for (int k = 0; k < n; k += U) {
        u32x4_t x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const u32x4_t*>((const T*)a.dx + (int64_t)list[min(k + u, n - 1)] * a.H + c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float o[VN];
            Vec<T>::load(reinterpret_cast<const T*>(&x[u]), o);
#pragma unroll
            for (int e = 0; e < VN; ++e) s[e] += k + u < n ? o[e] : 0.f;
        }
    }
    embed_out<T, MAIN>(a, t, c, s, old);
}

// workspace: the order (twice where spans have to be merged), then the parts
struct EmbedWs {
    size_t order, part, total;
    EmbedWs(int H, int n) {
        n = n > 0 ? n : 1;
        order = align_up((size_t)n * 4, 256);
        part = order * (n > SPAN ? 4 : 2);
        total = part + align_up((size_t)ceil_div(n, CH) * 2 * H * 4, 256);
    }
};

template <typename T, bool MAIN>
static hipError_t launch_embed_bwd(SumArgs a, SortArgs so, unsigned char* ws, hipStream_t st) {
    const EmbedWs L(a.H, a.n_max);
    const int n = a.n_max;
    so.tok = (int32_t*)ws;
    so.row = (int32_t*)(ws + L.order);
    so.spans = ceil_div(n, SPAN);
    if (!MAIN) {
        so.zero = (u32x4_t*)a.out;
        so.n_zero = (int64_t)a.V * a.H * (int64_t)sizeof(T) / 16;
    }
    const auto fill = [&](int threads) {        // blocks that clear the table beside those that put the rows in order
        const int64_t blocks = MAIN ? 0 : (so.n_zero + threads - 1) / threads;
        return (int)(blocks < MAX_GRID / 2 ? blocks : MAX_GRID / 2);
    };
    if (n <= FEW_ROWS) {
        if (!MAIN) embed_rank_kernel<<<fill(RANK_THREADS), RANK_THREADS, 0, st>>>(so, 0);      // clears the table
        if (n > 0) embed_few_kernel<T, MAIN><<<n * ceil_div(a.H / Vec<T>::N, 256), 256, 0, st>>>(a, so.tokens, so.idx);
        return hipGetLastError();
    }
    if (n <= SPAN) {
        const int rank_blocks = ceil_div(n, RANK_ROWS), grid = rank_blocks + fill(RANK_THREADS);
        embed_rank_kernel<<<grid, RANK_THREADS, 0, st>>>(so, rank_blocks);
    } else {
        static std::atomic<uint64_t> lds_ok{0};
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&embed_sort_kernel), SORT_LDS, lds_ok);
        if (e != hipSuccess) return e;
        embed_sort_kernel<<<so.spans + fill(SORT_THREADS), SORT_THREADS, SORT_LDS, st>>>(so);
    }
    a.tok = so.tok;
    a.row = so.row;
    if (so.spans > 1) {
        int32_t *tok = (int32_t*)(ws + 2 * L.order), *row = (int32_t*)(ws + 3 * L.order);
        embed_merge_kernel<<<ceil_div(n, 256) < MAX_GRID ? ceil_div(n, 256) : MAX_GRID, 256, 0, st>>>(a.tok, a.row, n, a.n_dev, tok, row);
        a.tok = tok;
        a.row = row;
    }
    a.part = (float*)(ws + L.part);
    const int vpr = a.H / Vec<T>::N, chunks = ceil_div(n, CH);
    const auto blocks = [&](int nt) { const int64_t u = (int64_t)chunks * ((vpr + nt - 1) / nt); return (int)(u < MAX_GRID ? u : MAX_GRID); };
    if (vpr <= 64) embed_sum_kernel<T, 64, MAIN><<<blocks(64), 64, 0, st>>>(a);
    else if (vpr <= 128) embed_sum_kernel<T, 128, MAIN><<<blocks(128), 128, 0, st>>>(a);
    else embed_sum_kernel<T, 256, MAIN><<<blocks(256), 256, 0, st>>>(a);
    if (chunks > 1) {
        const int64_t waves = (int64_t)(chunks - 1) * ((a.H + 255) / 256), blocks = (waves + 3) / 4, most = 16 * compute_units();
        embed_join_kernel<T, MAIN><<<(int)(blocks < most ? blocks : most), 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace cf

using namespace cf;

static cf_status embed_sizes(int32_t V, int32_t H, int32_t dtype) {
    if (dtype != CF_BF16 && dtype != CF_F32) return CF_ERR_DTYPE;
    if (V <= 0 || V > (1 << 30) || H <= 0 || H > (1 << 20) || H % (dtype == CF_F32 ? 4 : 8) != 0) return CF_ERR_SHAPE;
    return CF_OK;
}

extern "C" {

cf_status cf_embed_fwd(const void* table, int32_t V, int32_t H, int32_t dtype, const int64_t* tokens, int64_t n, float scale, void* out,
                       cf_stream stream) {
    if (!table || !tokens || !out) return CF_ERR_NULL;
    const cf_status ok = embed_sizes(V, H, dtype);
    if (ok != CF_OK) return ok;
    if (n < 0 || n > ((int64_t)1 << 40) / H || !(scale - scale == 0.f)) return CF_ERR_SHAPE;
    if (off_by(table, 16) || off_by(out, 16) || off_by(tokens, 8)) return CF_ERR_SHAPE;
    const uint64_t row = (uint64_t)H * dtype_size(dtype);
    if (ranges_meet(out, n * row, table, V * row)) return CF_ERR_SHAPE;
    if (n == 0) return CF_OK;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (dtype == CF_F32) launch_embed_fwd<float>(table, tokens, n, V, H, scale, out, st);
    else launch_embed_fwd<bf16_t>(table, tokens, n, V, H, scale, out, st);
    return hipGetLastError() == hipSuccess ? CF_OK : CF_ERR_HIP;
}

size_t cf_embed_bwd_workspace_bytes(int32_t H, int32_t max_kept) {
    if (H <= 0 || H > (1 << 20) || max_kept < 0 || max_kept > (1 << 30)) return 0;
    return EmbedWs(H, max_kept).total;
}

cf_status cf_embed_bwd(const int64_t* tokens, const void* dx_kept, int32_t V, int32_t H, int32_t dtype, const int32_t* idx,
                       const int32_t* n_kept_dev, int32_t max_kept, float scale, void* dtable, int32_t main_grad, void* ws, size_t ws_bytes,
                       cf_stream stream) {
    if (!tokens || !dx_kept || !dtable) return CF_ERR_NULL;
    const cf_status ok = embed_sizes(V, H, dtype);
    if (ok != CF_OK) return ok;
    if (max_kept < 0 || max_kept > (1 << 30) || (main_grad != 0 && main_grad != 1) || !(scale - scale == 0.f)) return CF_ERR_SHAPE;
    if (off_by(dx_kept, 16) || off_by(dtable, 16) || off_by(tokens, 8) || off_by(idx, 4) || off_by(n_kept_dev, 4)) return CF_ERR_SHAPE;
    const uint64_t es = dtype_size(dtype);
    if (ranges_meet(dtable, (uint64_t)V * H * (main_grad ? 4 : es), dx_kept, (uint64_t)max_kept * H * es)) return CF_ERR_SHAPE;
    if (!ws || off_by(ws, 256) || ws_bytes < cf_embed_bwd_workspace_bytes(H, max_kept)) return CF_ERR_WORKSPACE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    int passes = 0;
    for (int64_t v = V; v > 0; v >>= DIGIT_BITS) ++passes;
    SumArgs a{nullptr, nullptr, n_kept_dev, max_kept, V, H, dx_kept, scale, dtable, nullptr};
    SortArgs so{tokens, idx, n_kept_dev, max_kept, V, passes, nullptr, nullptr, 0, nullptr, 0};
    unsigned char* w = (unsigned char*)ws;
    hipError_t e;
    if (dtype == CF_F32) e = main_grad ? launch_embed_bwd<float, true>(a, so, w, st) : launch_embed_bwd<float, false>(a, so, w, st);
    else e = main_grad ? launch_embed_bwd<bf16_t, true>(a, so, w, st) : launch_embed_bwd<bf16_t, false>(a, so, w, st);
    return e == hipSuccess ? CF_OK : CF_ERR_HIP;
}

}  // extern "C"
