// Losses of kept tokens and their gradient towards the logits.  A block takes a row; one pass gives the running maximum and sum of its
// softmax, a second one, which needs both, the gradient.  HBM-bound: the kept rows of the logits in, the gradient out, if the row stays in registers
// between the passes; two exponentials an element are not far from what bounds it either.
#include <math.h>

#include "common.h"
#include "loss_row.h"

namespace cf {

// 16 bytes at an address that need only be aligned to an element: rows of an odd vocabulary start anywhere
typedef unsigned Bytes16 __attribute__((ext_vector_type(4), aligned(2)));

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
// What a block knows of a row apart from its logits.  The same for all its threads, which the compiler cannot know of what it loads:
// these go through the scalar path, apart from the vectors in flight (nothing in them is written during the kernel before it is read).
template <typename U> __device__ __forceinline__ U scalar_load(const U* p) {
    return *(const __attribute__((address_space(4))) U*)(uintptr_t)p;
}
template <typename T> __device__ __forceinline__ float scalar_load_f32(const void* base, int64_t i);
template <> __device__ __forceinline__ float scalar_load_f32<float>(const void* base, int64_t i) { return scalar_load((const float*)base + i); }
template <> __device__ __forceinline__ float scalar_load_f32<bf16_t>(const void* base, int64_t i) {
    const uintptr_t at = (uintptr_t)base + 2 * i;       // the dword around it
    const unsigned u = scalar_load((const unsigned*)(at & ~(uintptr_t)3));
    return __uint_as_float((at & 2) ? u & 0xFFFF0000u : u << 16);
}
template <typename T> __device__ __forceinline__ void find_row(const LossArgs& a, int j, RowHead& r) {
    r.row = a.idx != nullptr ? scalar_load(a.idx + j) : j;
    r.l = (const T*)a.logits + (int64_t)r.row * a.stride;
}
template <typename T> __device__ __forceinline__ void load_head(const LossArgs& a, RowHead& r) {
    const int64_t y = scalar_load(a.targets + r.row);
    r.w = a.weights != nullptr ? scalar_load(a.weights + r.row) : 1.f;
    r.old = r.ref = r.adv = 0.f;
    if (a.policy) {
        r.old = scalar_load(a.old_logp + r.row);
        r.adv = scalar_load(a.adv + r.row);
        if (a.ref_logp != nullptr) r.ref = scalar_load(a.ref_logp + r.row);
    }
    r.y = y >= 0 && y < a.V && r.w != 0.f ? (int)y : -1;
    r.ly = scalar_load_f32<T>(r.l, r.y < 0 ? 0 : r.y);
}
// One exponential of a softmax, 2^(k*(x - m)).  For fp32 logits (EXACT) the roundings of k*(x - m) and of k itself, up to 2^-19 of a small
// probability, are carried along and multiplied in; a bf16 gradient has 2^-8.
struct Expo {
    float m, k, klo;
};
template <bool EXACT> __device__ __forceinline__ float expo(const Expo& a, float x) {
    const float d = x - a.m, hi = d * a.k, e = __builtin_amdgcn_exp2f(hi);
    if (!EXACT) return e;
    const float lo = fmaf(d, a.klo, fmaf(d, a.k, -hi));
    return fmaf(e, hi > -200.f ? lo * 0.6931471805599453f : 0.f, e);       // behind a mask hi may be -inf, and lo NaN
}

// Maximum and sum of the block's threads: afterwards s is with respect to the common m
template <int WAVES> __device__ __forceinline__ void block_softmax(float k, float& m, float& s, float (&red)[2 * WAVES]) {
    float bm = m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) bm = fmaxf(bm, __shfl_xor(bm, o, 64));
    s = wave_sum(s * __builtin_amdgcn_exp2f((m - bm) * k));
    if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6] = bm; red[WAVES + (threadIdx.x >> 6)] = s; }
    __syncthreads();
    m = red[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) m = fmaxf(m, red[i]);
    s = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) s += red[WAVES + i] * __builtin_amdgcn_exp2f((red[i] - m) * k);
}

// The gradient's factors: neg times an exponential, at_y at the target.  `writes`: the thread that leaves what the row gives.
struct RowEnd {
    float neg, at_y;
};
__device__ __forceinline__ RowEnd row_end(const LossArgs& a, const RowHead& r, int j, float m, float s, float inv_norm, bool writes) {
    float lp = 0.f;
    RowLoss rl{make_float4(0.f, 0.f, 0.f, 0.f), 0.f};
    if (r.live()) {
        lp = (r.ly - m) * a.scale - logf(s);
        rl = row_loss(a, r, lp, inv_norm);
    }
    if (writes) {
        if (a.logp != nullptr) a.logp[j] = lp;
        a.terms[j] = rl.terms;
    }
    const float cs = rl.coef * a.scale;
    return RowEnd{-cs / s, -cs * expm1f(lp)};
}

// A row read twice, with no bound on its length
template <typename T, int NT> __device__ __forceinline__ void stream_row(const LossArgs& a, const RowHead& r, int j, float inv_norm, float (&red)[NT / 32]) {
    constexpr int VN = Vec<T>::N, WAVES = NT / 64, U = 4;          // vectors whose loads a thread has in flight
    constexpr bool EXACT = VN == 4;
    const int tid = threadIdx.x, V = a.V, nv = V / VN;
    const T* l = (const T*)r.l;
    Expo ex{-3.402823466e38f, a.k, a.klo};
    float s = 0.f;
    if (r.live()) {
        auto take = [&](const float (&x)[VN]) {
            float t = ex.m;
#pragma unroll
            for (int e = 0; e < VN; ++e) t = fmaxf(t, x[e]);
            s *= __builtin_amdgcn_exp2f((ex.m - t) * ex.k);
            ex.m = t;
#pragma unroll
            for (int e = 0; e < VN; ++e) s += expo<EXACT>(ex, x[e]);
        };
        for (int v = tid; v < nv; v += U * NT) {
            Bytes16 b[U];
#pragma unroll
            for (int u = 0; u < U; ++u) b[u] = reinterpret_cast<const Bytes16*>(l)[min(v + u * NT, nv - 1)];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * NT >= nv) break;
                float x[VN];
                widen<T>(b[u], x);
                take(x);
            }
        }
        if (int c = nv * VN + tid; c < V) {
            float x[VN];
            x[0] = to_f32<T>(l[c]);
#pragma unroll
            for (int e = 1; e < VN; ++e) x[e] = -INFINITY;
            take(x);
        }
        block_softmax<WAVES>(ex.k, ex.m, s, red);
    }
    const RowEnd end = row_end(a, r, j, ex.m, s, inv_norm, threadIdx.x == 0);
    if (a.dlogits == nullptr) return;
    T* dl = (T*)a.dlogits + (int64_t)j * a.dstride;
    for (int v = tid; v < nv; v += U * NT) {
        Bytes16 b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) b[u] = reinterpret_cast<const Bytes16*>(l)[min(v + u * NT, nv - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = v + u * NT;
            if (at >= nv) break;
            float x[VN];
            widen<T>(b[u], x);
#pragma unroll
            for (int e = 0; e < VN; ++e) x[e] = !r.live() ? 0.f : at * VN + e == r.y ? end.at_y : end.neg * expo<EXACT>(ex, x[e]);
            __builtin_nontemporal_store(narrow<T>(x), reinterpret_cast<Bytes16*>(dl) + at);
        }
    }
    if (int c = nv * VN + tid; c < V)
        dl[c] = narrow_one<T>(!r.live() ? 0.f : c == r.y ? end.at_y : end.neg * expo<EXACT>(ex, to_f32<T>(l[c])));
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void token_loss_stream_kernel(LossArgs a) {
    __shared__ float red[NT / 32];
    const int n_rows = live_rows(a.n_max, a.n_dev), j = a.first + (int)blockIdx.x;
    if (j >= n_rows) return;
    RowHead r;
    find_row<T>(a, j, r);
    load_head<T>(a, r);
    stream_row<T, NT>(a, r, j, 1.f / (a.norm != 0.f ? a.norm : (float)n_rows), red);
}

// A row in a block's registers, NV vectors of 16 bytes a thread, so that it is read once.  The block walks through rows, and each vector of the next
// row is asked for as soon as its register has given its part of the gradient (or of the sum, without a gradient), or BURST of them together: reads, arithmetic
// and writes of neighbouring rows overlap.  4096 of 8192 rows of 128256 bf16 logits: 2.1 GB in 382 us, 5.5 TB/s where a copy of 1 GiB reaches 6.2; read
// twice it took 601.  4096 rows of 32000 102 us (126), 701 of 50257 fp32 logits 56 us (87).  Arithmetic does not bound it: with its exponentials left out
// it took 402 of 405 before the bursts.
// The gradient is written past the caches: 406 against 417 us, 102 against 110; with the two products of a [V, 2048] head behind it, 64 to 2048 rows
// of 32000 take 0.97 to 1.00 of the time, 1024 of 128256 0.995, and 4096 of 32000, which just fit the last cache, 1.03.
// Four vectors a thread leave registers for eight waves a SIMD: 8192 rows of 8000 56 -> 49 us, 16384 of 1000 fp32 42 -> 36; eight vectors do not
// (8192 rows of 16000 105 -> 115).  Rows that start on odd elements cost 1.1 (4096 x 50257 and 50264: 190 and 171 us, without gradient 102 and 79): their
// 16-byte loads lie between dwords.
// Keeps a vector as it is stored, and the arithmetic where it stands: widened values of one pass are not to be kept for the next one.
__device__ __forceinline__ void hold(Bytes16& b) { asm volatile("" : "+v"(b)); }
__device__ __forceinline__ void hold(float& a, float& b) { asm volatile("" : "+v"(a), "+v"(b)); }

// A vector at a scalar address and a lane's offset from it.  Without the empty statement the lane's part is added up in 64 bits for each vector.
__device__ __forceinline__ Bytes16* vector_at(const void* base, unsigned offset) {
    uintptr_t p = (uintptr_t)base;
    asm("" : "+s"(p));
    return (Bytes16*)((__attribute__((address_space(1))) char*)p + offset);
}

template <typename T, int NT, int NV, int BURST, bool GRAD>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(NV <= 4 ? 8 : 4, 8))) void token_loss_kernel(LossArgs a) {
    constexpr int VN = Vec<T>::N, WAVES = NT / 64;
    // The launch takes this kernel for rows of more than FULL * NT vectors: up to there every lane has one.  Behind, a vector that no lane has is skipped,
    // and lanes behind the last one do what its owner does.  No access is conditional but for that: what is in flight is counted, and
    // a count that hangs on a branch is waited for as if the branch had not been taken.
    constexpr int FULL = NV <= 4 ? 0 : NV - 4;
    constexpr bool EXACT = VN == 4;
    __shared__ float red[2 * WAVES];
    __shared__ float ends[3];
    const int n_rows = live_rows(a.n_max, a.n_dev), tid = threadIdx.x, V = a.V, nv = V / VN, ct = nv * VN + tid;
    int j = blockIdx.x, jn;
    if (j >= n_rows) return;
    const float inv_norm = 1.f / (a.norm != 0.f ? a.norm : (float)n_rows);
    Bytes16 x[NV];
    auto at = [&](int i) __attribute__((always_inline)) { return (unsigned)(i < FULL ? tid : min(tid, nv - 1 - i * NT)) * 16u; };
    auto load = [&](const void* l, int i) __attribute__((always_inline)) { return *vector_at((const char*)l + i * NT * 16, at(i)); };
    const int tail_at = min(ct, V - 1);         // the row's last elements, one a thread, as they are stored
    // the next row's; behind the last row all lanes ask for its first 16 bytes, over and over
    unsigned far = ~0u;
    auto load_next = [&](const void* l, int i) __attribute__((always_inline)) {
        return *vector_at((const char*)l + (far & (unsigned)(i * NT * 16)), at(i) & far);
    };
    RowHead r, rn;
    T xt;
    Expo ex{0.f, a.k, a.klo};
    float s, tail;
    // What the row needs apart from its vectors, and where the next one is; the threads' maximum and sum
    auto begin = [&]() __attribute__((always_inline)) {
        load_head<T>(a, r);
        rn = r;
        jn = j + (int)gridDim.x;
        if (jn < n_rows) find_row<T>(a, jn, rn);
        far = jn < n_rows ? ~0u : 0u;
        ex.m = -3.402823466e38f;
        s = 0.f;
        auto take = [&](const auto& o) __attribute__((always_inline)) {
            constexpr int N = sizeof(o) / sizeof(float);
            float t = ex.m;
#pragma unroll
            for (int e = 0; e < N; ++e) t = fmaxf(t, o[e]);
            s *= __builtin_amdgcn_exp2f((ex.m - t) * ex.k);
            ex.m = t;
#pragma unroll
            for (int e = 0; e < N; ++e) s += expo<EXACT>(ex, o[e]);
            hold(ex.m, s);
        };
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i >= FULL && i * NT >= nv) continue;
            float o[VN];
            hold(x[i]);
            widen<T>(x[i], o);
            if (i >= FULL && nv - i * NT < NT) {
#pragma unroll
                for (int e = 0; e < VN; ++e) o[e] = tid < nv - i * NT ? o[e] : -INFINITY;
            }
            take(o);
            if (!GRAD) x[i] = load_next(rn.l, i);
            __builtin_amdgcn_sched_barrier(0);
        }
        tail = ct < V ? to_f32<T>(xt) : -INFINITY;
        const float o1[1] = {tail};
        take(o1);
        if (!GRAD) xt = ((const T*)rn.l)[tail_at];
    };
    find_row<T>(a, j, r);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i < FULL || i * NT < nv) x[i] = load(r.l, i);
        __builtin_amdgcn_sched_barrier(0);
    }
    xt = ((const T*)r.l)[tail_at];
    begin();            // not the loop's: there the loads stand between stores
    for (;;) {
        // over the wave; the first wave adds up the waves and ends the row
        float m = ex.m;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        s = wave_sum(s * __builtin_amdgcn_exp2f((ex.m - m) * ex.k));
        if ((tid & 63) == 0) { red[tid >> 6] = m; red[WAVES + (tid >> 6)] = s; }
        __syncthreads();
        if (tid < 64) {
            const float wm = red[tid & (WAVES - 1)];
            m = wm;
            s = red[WAVES + (tid & (WAVES - 1))];
#pragma unroll
            for (int o = WAVES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
            s *= __builtin_amdgcn_exp2f((wm - m) * ex.k);
#pragma unroll
            for (int o = WAVES / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
            const RowEnd end = row_end(a, r, j, m, s, inv_norm, tid == 0);
            if (tid == 0) { ends[0] = m; ends[1] = end.neg; ends[2] = end.at_y; }
        }
        __syncthreads();
        if (GRAD) {
            ex.m = ends[0];
            const float neg = ends[1], at_y = ends[2];
            auto grad = [&](float v) __attribute__((always_inline)) { return neg * expo<EXACT>(ex, v); };
            char* dl = (char*)((T*)a.dlogits + (int64_t)j * a.dstride);
            const unsigned yv = (unsigned)(r.y >> (VN == 8 ? 3 : 2)) * 16u;
            const int ye = r.y & (VN - 1);
            if (ct < V) ((T*)dl)[ct] = narrow_one<T>(!r.live() ? 0.f : ct == r.y ? at_y : grad(tail));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i < FULL || i * NT < nv) {
                    Bytes16 g;
                    hold(x[i]);
                    if (r.live()) {
                        float o[VN];
                        widen<T>(x[i], o);
#pragma unroll
                        for (int e = 0; e < VN; ++e) o[e] = grad(o[e]);
                        if (at(i) == yv - i * NT * 16) {
#pragma unroll
                            for (int e = 0; e < VN; ++e) o[e] = e == ye ? at_y : o[e];
                        }
                        g = narrow<T>(o);
                        hold(g);
                    } else {
                        g = Bytes16{0u, 0u, 0u, 0u};
                        hold(g);
                    }
                    x[i] = g;
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (i % BURST == BURST - 1 || i == NV - 1) {
#pragma unroll
                    for (int z = i / BURST * BURST; z <= i; ++z)
                        if (z < FULL || z * NT < nv) __builtin_nontemporal_store(x[z], vector_at(dl + z * NT * 16, at(z)));
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int z = i / BURST * BURST; z <= i; ++z)
                        if (z < FULL || z * NT < nv) x[z] = load_next(rn.l, z);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            xt = ((const T*)rn.l)[tail_at];
        }
        if (jn >= n_rows) return;
        j = jn;
        r = rn;
        begin();
    }
}

// stats = sums of the rows' terms over the live rows, in fp64 and in fixed order, over norm
__global__ __launch_bounds__(1024) void loss_stats_kernel(const float4* __restrict__ terms, int n_max, const int32_t* __restrict__ n_dev,
                                                         float norm, float* __restrict__ stats) {
    __shared__ double red[16][4];
    const int n_rows = live_rows(n_max, n_dev);
    double s[4] = {0., 0., 0., 0.};
#pragma unroll 4
    for (int j = threadIdx.x; j < n_rows; j += 1024) {
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
        double t = 0.;
#pragma unroll
        for (int i = 0; i < 16; ++i) t += red[i][threadIdx.x];
        const double by = norm != 0.f ? (double)norm : (double)(n_rows > 0 ? n_rows : 1);
        stats[threadIdx.x] = (float)(t / by);
    }
}

void launch_loss_stats(const float4* terms, int n_max, const int32_t* n_dev, float norm, float* stats, hipStream_t st) {
    loss_stats_kernel<<<1, 1024, 0, st>>>(terms, n_max, n_dev, norm, stats);
}

template <typename T, int NT, int NV> static void launch_rows(const LossArgs& a, hipStream_t st) {
    const int resident = compute_units() * (1024 / NT) * (NV <= 4 ? 2 : 1), grid = a.n_max < resident ? a.n_max : resident;
    if (a.dlogits == nullptr) { token_loss_kernel<T, NT, NV, 1, false><<<grid, NT, 0, st>>>(a); return; }
    if constexpr (NT == 1024) {
        // Whole rows at once: a block that has a CU to itself computes a row's gradient into its registers, writes all of it and asks for all of the next
        // row.  What is open in memory at one time then lies closer together: 4096 x 128256 bf16 403 -> 383 us, x 151936 485 -> 452, 2048 x 50257 fp32 176
        // -> 169.  Not where rows lie between dwords, whose parts of a line the caches would have to hold longer (2048 x 128257 244 -> 256), and not for
        // less than three rows a block (512 x 128256 50.7 -> 51.8).
        if ((uintptr_t)a.dlogits % 4 == 0 && (a.dstride * sizeof(T)) % 4 == 0 && (int64_t)a.n_max > 2 * (int64_t)grid) {
            token_loss_kernel<T, NT, NV, NV, true><<<grid, NT, 0, st>>>(a);
            return;
        }
    }
    token_loss_kernel<T, NT, NV, 1, true><<<grid, NT, 0, st>>>(a);
}

// The smallest block whose registers hold a row.  A function of the vocabulary and the type alone: a row's sums, and its logp, are
// added up in the same order in every call.
template <typename T> static void launch_token_loss(LossArgs& a, hipStream_t st) {
    const int nv = a.V / Vec<T>::N;
    if (nv < 1 || nv > 1024 * 20) {
        for (; a.first < a.n_max; a.first += MAX_GRID)
            token_loss_stream_kernel<T, 1024><<<a.n_max - a.first < MAX_GRID ? a.n_max - a.first : MAX_GRID, 1024, 0, st>>>(a);
    } else if (nv <= 256 * 4) launch_rows<T, 256, 4>(a, st);
    else if (nv <= 256 * 8) launch_rows<T, 256, 8>(a, st);
    else if (nv <= 256 * 12) launch_rows<T, 256, 12>(a, st);
    else if (nv <= 256 * 16) launch_rows<T, 256, 16>(a, st);
    else if (nv <= 512 * 12) launch_rows<T, 512, 12>(a, st);
    else if (nv <= 512 * 16) launch_rows<T, 512, 16>(a, st);
    else if (nv <= 1024 * 12) launch_rows<T, 1024, 12>(a, st);
    else if (nv <= 1024 * 16) launch_rows<T, 1024, 16>(a, st);
    else launch_rows<T, 1024, 20>(a, st);
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
    const cf_status ok = loss_desc_check(desc, old_logp, ref_logp, advantages, max_kept);
    if (ok != CF_OK) return ok;
    const int64_t ls = logits_stride ? logits_stride : desc->V, ds = dlogits_stride ? dlogits_stride : desc->V;
    if (ls < desc->V || (dlogits && ds < desc->V)) return CF_ERR_SHAPE;
    const size_t e = dtype_size(desc->dtype);
    const auto off = [](const void* p, size_t a) { return p && (uintptr_t)p % a != 0; };
    if (off(logits, e) || off(dlogits, e) || off(targets, 8)) return CF_ERR_SHAPE;
    for (const void* p : {(const void*)old_logp, (const void*)ref_logp, (const void*)advantages, (const void*)weights, (const void*)idx,
                          (const void*)n_kept_dev, (const void*)logp, (const void*)stats})
        if (off(p, 4)) return CF_ERR_SHAPE;
    // a row would be written before another block has read it
    if (dlogits == logits && (idx || ls != ds)) return CF_ERR_SHAPE;
    if (dlogits && dlogits != logits && !idx && max_kept > 0) {
        const uintptr_t l0 = (uintptr_t)logits, d0 = (uintptr_t)dlogits;
        const uint64_t ln = ((uint64_t)(max_kept - 1) * ls + desc->V) * e, dn = ((uint64_t)(max_kept - 1) * ds + desc->V) * e;
        if (l0 < d0 + dn && d0 < l0 + ln) return CF_ERR_SHAPE;
    }
    if (!ws || off(ws, 16) || ws_bytes < cf_token_loss_workspace_bytes(max_kept)) return CF_ERR_WORKSPACE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    LossArgs a = loss_args(desc, targets, old_logp, ref_logp, advantages, weights, idx, n_kept_dev, max_kept, logp);
    a.logits = logits; a.stride = ls;
    a.dlogits = dlogits; a.dstride = ds;
    a.terms = (float4*)ws;
    if (max_kept > 0) desc->dtype == CF_F32 ? launch_token_loss<float>(a, st) : launch_token_loss<bf16_t>(a, st);
    if (stats) launch_loss_stats((const float4*)ws, max_kept, n_kept_dev, desc->norm, stats, st);
    return hipGetLastError() == hipSuccess ? CF_OK : CF_ERR_HIP;
}

}  // extern "C"
