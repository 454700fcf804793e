// What follows the last layer of a node classifier or of an entity ranker: per row of scores z [N,C]
//   lse = log sum_c exp z_c,  logp = z_label - lse,  H = -sum_c p_c log p_c (p = exp(z - lse)),  the k best classes and their log p
// in one pass over the scores, and the gradient of logp and H
//   dz_c = dlogp ([c = label] - p_c) - dH p_c (log p_c + H).
//
// Running statistics of a part of a row: m (largest score), s = sum of exp(z - m) over all classes BUT one of those at m, and
// t = sum of exp(z - m) (z - m).  Then lse = m + log1p(s) and H = log1p(s) - t / (1 + s): without the leading 1 in the sum, a
// row whose best class is nearly sure keeps the digits of its small log p and entropy.  Two parts are joined by scaling the one
// with the smaller maximum, whose own maximum counts again: exp(m1 - m2) (s1 + 1).
// The k best: keys of (score, lower index first) that are all different.  A floor of the k-th best, from the threads' largest scores, leaves
// few chunks to look at again, and what reaches it in them is sorted over the lanes of a warp; where too few or too many do, every class is
// offered to a sorted list (log_probs_kernel).  Rows of few classes: log_probs_few_kernel.
#include <cooperative_groups.h>

#include <type_traits>

#include "tc_common.cuh"

namespace gnn {

constexpr int LP_TOP = 32;            // classes listed at most: a lane each
// Rows up to here by a warp, longer ones by a block.  By a warp / by a block, fp32, no list: 20,000 rows of 300 classes 13.5 / 66 us, of 1000 19.9 / 71, of
// 2000 39 / 90; five best 30 / 112, 68 / 117, 93 / 143; but 64 rows of 1000, five best: 11.0 / 4.1.  (Many rows would gain from a
// higher border, few rows from a lower one.)
constexpr int LP_WARP_CLASSES = 1024;
constexpr int LP_SLOT = 56;           // of allow_big_smem: four of them
constexpr int LP_CLUSTER = 8;         // parts of a row that a cluster of blocks joins; more leave theirs in the workspace

__device__ __forceinline__ float lp_exp(float d) {  // exp of d <= 0: 2^(d log2 e); the error of the product reaches what is below e^-10 by 1e-6 of it
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(d * 1.4426950408889634f));
    return e;
}

struct LpStats {
    float m, s, t;
    __device__ __forceinline__ void clear() { m = -INFINITY; s = 0.f; t = 0.f; }
    // z <= m, or not a number (which then shows in s)
    __device__ __forceinline__ void add(float z, float base) {
        const float d = z - base, e = lp_exp(d);
        s += e;
        t = fmaf(e, fmaxf(d, -1000.f), t);  // e = 0 where d = -inf
    }
    __device__ __forceinline__ void join(const LpStats& o) {
        if (o.m > m) {
            const LpStats mine = *this;
            *this = o;
            fold(mine);
        } else {
            fold(o);
        }
    }
    __device__ __forceinline__ void fold(const LpStats& o) {  // o.m <= m
        if (o.m == -INFINITY) { s += o.s; return; }  // nothing in it, or not numbers only
        const float d = o.m - m, f = lp_exp(d), c = f * (o.s + 1.f);
        s += c;
        t += fmaf(fmaxf(d, -1000.f), c, f * o.t);  // d = -inf: times 0
    }
};

// largest key = best: score above, lower index first; 0: no class.  -0 counts as 0, what is not a number comes last.
__device__ __forceinline__ uint64_t lp_key(float z, uint32_t c) {
    const uint32_t b = __float_as_uint(z + 0.f);
    const uint32_t v = z != z ? 1u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return (uint64_t)v << 32 | (0xFFFFFFFFu - c);
}
__device__ __forceinline__ uint32_t lp_class(uint64_t key) { return 0xFFFFFFFFu - (uint32_t)key; }
__device__ __forceinline__ float lp_score(uint64_t key) {
    const uint32_t v = (uint32_t)(key >> 32);
    return v == 1u ? __uint_as_float(0x7FC00000u) : __uint_as_float((v & 0x80000000u) ? v & 0x7FFFFFFFu : ~v);
}

// Sorting over the lanes of a warp, largest in lane 0 (bitonic: 15 exchanges; a merge of two sorted lists into the best 32: 6)
template <typename V>
__device__ __forceinline__ V lp_exchange(V v, int o, bool keep_larger) {
    const V w = __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return (v > w) == keep_larger ? v : w;
}
template <typename V>
__device__ __forceinline__ V lp_sort(V v, int lane) {
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
        for (int o = size / 2; o > 0; o >>= 1) v = lp_exchange(v, o, ((lane & o) == 0) == ((lane & size) == 0 || size == 32));
    return v;
}
template <typename V>
__device__ __forceinline__ V lp_merge(V a, V b, int lane) {  // both sorted
    const V r = __shfl_sync(0xFFFFFFFFu, b, 31 - lane);
    a = a > r ? a : r;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = lp_exchange(a, o, (lane & o) == 0);
    return a;
}

// the k best so far, lane j the j-th; last: the worst of them (0: not full)
struct LpTop {
    uint64_t key, last;
    __device__ __forceinline__ void clear() { key = 0; last = 0; }
    __device__ __forceinline__ void insert(uint64_t cand, int k, int lane) {  // the same cand in all lanes
        if (cand <= last) return;
        const uint64_t up = __shfl_up_sync(0xFFFFFFFFu, key, 1);
        if (cand > key) key = lane > 0 && cand > up ? up : cand;
        last = __shfl_sync(0xFFFFFFFFu, key, k - 1);
    }
    // one candidate per lane
    __device__ __forceinline__ void offer(uint64_t cand, int k, int lane) {
        uint32_t who = __ballot_sync(0xFFFFFFFFu, cand > last);
        while (who) {
            const int l = __ffs(who) - 1;
            who &= who - 1;
            insert(__shfl_sync(0xFFFFFFFFu, cand, l), k, lane);
        }
    }
};
// the best of n keys in shared memory, by one warp
__device__ __forceinline__ uint64_t lp_best_of(const uint64_t* keys, int n, int lane) {
    uint64_t best = 0;
    for (int i = 0; i < n; i += 32) best = lp_merge(best, lp_sort(i + lane < n ? keys[i + lane] : 0, lane), lane);
    return best;
}

// Running sums of one thread: r = m log2(e) rounded, s = sum of 2^(z log2(e) - r) over all of its classes, t the same weighted by the
// exponent.  Two classes at a time (packed fp32 instructions).  z log2(e) - r is one rounding off whatever m is; what r itself is off
// by (1 at most up to |m| = 2^24) is taken out at the end.  A row whose largest score is beyond FAR is summed again from its threads'
// maxima, the exponent as (z - m) log2(e): exact there, an instruction more per pair.  What the threads' first sums have to be
// until then is finite, since masks (-1e9 or -1e30, say) may come before the scores of a nearer row: up to 2^30 r is off by 64 at most;
// beyond, where m log2(e) could be off by more than an exponent holds, neighbouring numbers are 128 apart: 2^(z - m) tells as well who is at
// m, and all others are 0.
struct LpRun {
    float m, r;
    float2 k, minus;  // the factor, and -r (from_maximum: -m), twice each
    float2 s, t;
    bool exact;       // from_maximum
    static constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f, FAR = 16777216.f, LIMIT = 1073741824.f;
    __device__ __forceinline__ void clear() {
        m = -INFINITY; r = 0.f; exact = false;
        k = make_float2(LOG2E, LOG2E);
        minus = s = t = make_float2(0.f, 0.f);
    }
    static __device__ __forceinline__ float exp2_(float u) {
        float e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u));
        return e;
    }
    // the maximum becomes v > m
    __device__ __forceinline__ void raise(float v) {
        const float factor = fabsf(v) > LIMIT ? 1.f : LOG2E;
        const bool none = m == -INFINITY || factor != k.x;  // of the sums so far (another factor: v is 128 above m at least)
        k.x = k.y = factor;
        // (rounded as r is before it is taken from r: in one instruction with that the sums would stand for another r than the next ones')
        const float q = __fmul_rn(v, k.x), d = fmaxf(r - q, -2000.f), f = none ? 0.f : exp2_(d);
        t = none ? make_float2(0.f, 0.f) : make_float2(f * fmaf(d, s.x, t.x), f * fmaf(d, s.y, t.y));
        s = make_float2(f * s.x, f * s.y);  // (not a number stays one)
        m = v;
        r = q;
        minus = make_float2(-q, -q);
    }
    // the sums anew, by add<true>, for the largest score (or -inf: there is none)
    __device__ __forceinline__ void from_maximum(float v) {
        clear();
        m = v;
        exact = true;
        if (v > -INFINITY) minus = make_float2(-v, -v);
    }
    // two scores, neither above m; -inf: 2^-inf = 0 times a finite exponent
    template <bool EXACT>
    __device__ __forceinline__ void add(float a, float b) {
        const float2 z = make_float2(a, b), u = EXACT ? fma2(add2(z, minus), make_float2(LOG2E, LOG2E), make_float2(0.f, 0.f)) : fma2(z, k, minus);
        const float2 e = make_float2(exp2_(u.x), exp2_(u.y));
        s = add2(s, e);
        t = fma2(e, make_float2(fmaxf(u.x, -2000.f), fmaxf(u.y, -2000.f)), t);
    }
    // taken_out: of the sums a class at m (the 1 that LpStats leaves out)
    __device__ __forceinline__ LpStats stats(bool taken_out = false) const {
        LpStats o;
        const float S = s.x + s.y;
        o.m = m;
        if (!(m > -INFINITY) || m == INFINITY) { o.s = S == S && m < INFINITY ? 0.f : __uint_as_float(0x7FC00000u); o.t = 0.f; return o; }
        const float off = exact ? 0.f : fmaf(m, k.x, -r), f = exp2_(-off);
        o.s = taken_out ? f * S : fmaf(f, S, -1.f);
        o.t = LN2 * f * fmaf(-off, S, t.x + t.y);
        return o;
    }
};

struct LpParams {
    const void* z;
    const int32_t* label;  // or nullptr
    int64_t N;
    int C, top;
    float *logp, *entropy, *lse, *lse_rest, *top_logp;  // each may be nullptr
    int32_t* top_idx;
    int parts;          // blocks per row (whole-block rows)
    float* stats;       // [N][parts][4] where parts > 1
    uint64_t* keys;     // [N][parts][top]
};

// lse = m + log1p(s), and what its rounding leaves out (exactly: the sum of two numbers in two)
__device__ __forceinline__ void lp_lse_out(const LpParams& P, int64_t row, float m, float tail, bool bad, bool none) {
    const float lse = bad ? __uint_as_float(0x7FC00000u) : none ? -INFINITY : m + tail;
    if (P.lse) P.lse[row] = lse;
    if (P.lse_rest) {
        const float b = lse - m;
        P.lse_rest[row] = bad || none ? 0.f : (m - (lse - b)) + (tail - b);
    }
}

// what a row answers, from its statistics (all lanes) and its best (a lane each)
template <typename T>
__device__ __forceinline__ void lp_finish(const LpParams& P, int64_t row, const LpStats& st, float z_label, uint64_t best, int lane) {
    const float nan = __uint_as_float(0x7FC00000u);
    const bool bad = st.s != st.s || st.m == INFINITY, none = st.m == -INFINITY;
    const float tail = log1pf(st.s);
    // z - lse as (z - m) - log1p(s): exact where z is the largest
    auto logp = [&](float z) { return bad ? nan : none || z == -INFINITY ? -INFINITY : (z - st.m) - tail; };
    if (lane == 0) {
        lp_lse_out(P, row, st.m, tail, bad, none);
        if (P.entropy) P.entropy[row] = bad ? nan : none ? 0.f : tail - st.t / (1.f + st.s);
        if (P.logp) {
            const int y = P.label[row];
            P.logp[row] = y >= 0 && y < P.C ? logp(z_label) : 0.f;
        }
    }
    if (lane < P.top) {
        P.top_idx[row * P.top + lane] = (int32_t)lp_class(best);
        P.top_logp[row * P.top + lane] = logp(lp_score(best));
    }
}

// Few classes, many rows: a thread per row.  A block's rows are consecutive in memory: they arrive by whole chunks and are handed
// over through shared memory, as they lie (words of a warp's rows then fall on one bank at most two at a time), or, where the
// number of classes is a multiple of four, in rows of an odd number of 16-byte words.
// The best: the largest of the groups' largest scores (eight classes each), then its group again in shared memory, where what is
// taken becomes NaN.  170,000 x 47, five best: by a warp per row 158 us, with a row's scores in registers, looked through for every
// class listed, 29 us; so 15.8 us (2.1 TB/s; half of all cycles issue).
constexpr int LP_ROWS = 128;  // of a block
constexpr int LP_FEW = 64;    // classes at most: NG groups of eight
__host__ __device__ constexpr int lp_few_stride(int C) { return C % 4 == 0 ? (C / 4 | 1) * 4 : C; }

template <typename T, int NG>
__global__ void __launch_bounds__(LP_ROWS)
log_probs_few_kernel(const LpParams P) {
    pdl_wait();
    constexpr int PER = Chunk<T>::N;
    extern __shared__ __align__(16) float sh_z[];  // [LP_ROWS][stride] and a chunk
    const int C = P.C, stride = lp_few_stride(C);
    const int64_t r0 = (int64_t)blockIdx.x * LP_ROWS;
    const int rows = (int)(P.N - r0 < LP_ROWS ? P.N - r0 : LP_ROWS);
    const T* const z = (const T*)P.z + r0 * C;  // on 16 bytes: LP_ROWS rows are
    const int elements = rows * C;
    constexpr int U = 4;  // chunks in flight per thread
    for (int e0 = (int)threadIdx.x * PER; e0 < elements; e0 += U * LP_ROWS * PER) {
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (e0 + u * LP_ROWS * PER + PER <= elements) v[u] = ld_16(z + e0 + u * LP_ROWS * PER);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = e0 + u * LP_ROWS * PER;
            float f[PER];
            if (e >= elements) break;
            if (e + PER <= elements) Chunk<T>::unpack(v[u], f);
            else
#pragma unroll
                for (int k = 0; k < PER; ++k) f[k] = e + k < elements ? (float)z[e + k] : 0.f;
#pragma unroll
            for (int k = 0; k < PER; k += 4) {  // (four lie in one row where rows are padded)
                const int at = stride == C ? e + k : e + k + (int)((unsigned)(e + k) / (unsigned)C) * (stride - C);
                *reinterpret_cast<float4*>(sh_z + at) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
            }
        }
    }
    __syncthreads();
    if ((int)threadIdx.x >= rows) return;
    const int64_t row = r0 + threadIdx.x;
    float* const mine = sh_z + threadIdx.x * stride;
    const float nan = __uint_as_float(0x7FC00000u);
    // groups of eight classes, the last may be cut: their largest
    const int full = C / 8;
    float gm[NG];
    float m = nan;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        gm[g] = nan;
        if (g < full) {
#pragma unroll
            for (int c = 0; c < 8; ++c) gm[g] = fmaxf(gm[g], mine[8 * g + c]);
        } else if (g == full) {
            for (int c = 8 * g; c < C; ++c) gm[g] = fmaxf(gm[g], mine[c]);
        }
        m = fmaxf(m, gm[g]);
    }
    // the first class at m (C: there is no number left); its group's next largest takes its place
    auto take = [&](float m) {
        int first = NG;
#pragma unroll
        for (int g = NG - 1; g >= 0; --g) first = gm[g] == m ? g : first;
        if (first == NG) return C;
        int at = C;
        float next = nan;
#pragma unroll
        for (int c = 7; c >= 0; --c) {
            const float x = 8 * first + c < C ? mine[8 * first + c] : nan;
            const bool hit = x == m;
            next = hit ? (at < C ? m : next) : fmaxf(next, x);  // an equal one stays
            at = hit ? 8 * first + c : at;
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) gm[g] = g == first ? next : gm[g];
        return at;
    };
    const int lead = take(m);
    // the sums without the leading class: at -inf meanwhile
    LpRun run;
    run.clear();
    if (m > -INFINITY) mine[lead] = -INFINITY;
    if (fabsf(m) > LpRun::FAR && fabsf(m) < INFINITY) {
        run.from_maximum(m);
        for (int c = 0; c < C; ++c) run.add<true>(mine[c], -INFINITY);
    } else {
        if (m > -INFINITY) run.raise(m);
        for (int g = 0; g < full; ++g)
#pragma unroll
            for (int c = 0; c < 8; c += 2) run.add<false>(mine[8 * g + c], mine[8 * g + c + 1]);
        for (int c = 8 * full; c < C; ++c) run.add<false>(mine[c], -INFINITY);
    }
    if (lead < C) mine[lead] = nan;  // taken
    const LpStats st = run.stats(true);
    const bool bad = st.s != st.s || st.m == INFINITY, none = st.m == -INFINITY;
    const float tail = log1pf(st.s);
    auto logp = [&](float x) { return bad ? nan : none || x == -INFINITY ? -INFINITY : (x - st.m) - tail; };
    lp_lse_out(P, row, st.m, tail, bad, none);
    if (P.entropy) P.entropy[row] = bad ? nan : none ? 0.f : tail - st.t / (1.f + st.s);
    if (P.logp) {
        const int y = P.label[row];
        P.logp[row] = y >= 0 && y < C ? logp(y == lead ? m : mine[y]) : 0.f;
    }
    for (int j = 0; j < P.top; ++j) {
        int at = lead;
        if (j > 0) {
            m = gm[0];
#pragma unroll
            for (int g = 1; g < NG; ++g) m = fmaxf(m, gm[g]);
            at = take(m);
            if (at < C) mine[at] = nan;
        }
        if (at == C) {  // numbers are used up: what is not one, in order
            const T* const orig = z + (int64_t)threadIdx.x * C;
            int skip = j;
            for (int c = 0; c < C; ++c) skip -= (float)orig[c] == (float)orig[c];
            for (int c = 0; c < C; ++c)
                if ((float)orig[c] != (float)orig[c] && skip-- == 0) at = c;
            m = nan;
        }
        P.top_idx[row * P.top + j] = at;
        P.top_logp[row * P.top + j] = logp(m);
    }
}

// The statistics of a warp's lanes joined, all lanes alike: every lane's sum scaled to the largest maximum, that of the first lane
// that has it without its own 1.
__device__ __forceinline__ void lp_join_lanes(LpStats& st, int lane) {
    float m = st.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    const bool lead = lane == __ffs(__ballot_sync(0xFFFFFFFFu, st.m == m)) - 1;  // m is a number or -inf: some lane has it
    const float d = st.m - m, f = lp_exp(d), c = f * (st.s + 1.f);  // a lane without classes: -inf - m (NaN where m is -inf as well: below)
    float s = st.m == -INFINITY ? 0.f * st.s : lead ? st.s : c;
    float t = st.m == -INFINITY ? 0.f : lead ? st.t : fmaf(fmaxf(d, -1000.f), c, f * st.t);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
    }
    st.m = m;
    st.s = s;
    st.t = t;
}
// ... and of the block's eight warps, joined by every warp
__device__ __forceinline__ LpStats lp_join_warps(const LpStats* sh, int lane) {
    LpStats st;
    st.clear();
    if (lane < 8) st = sh[lane];
    lp_join_lanes(st, lane);
    return st;
}

// largest of a chunk, what is not a number left out (NaN where there is none)
template <typename T>
__device__ __forceinline__ float lp_chunk_max(uint4 v) {
    if constexpr (Chunk<T>::N == 4) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    } else {
        auto larger = [](uint32_t a, uint32_t b) {
            uint32_t c;
            asm("max.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
            return c;
        };
        const uint32_t m = larger(larger(v.x, v.y), larger(v.z, v.w));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    }
}

// Rows by W warps (1: eight rows a block; 8: a row, or a part of one, per block), in one pass over the scores.
// The best classes: every thread keeps the largest score of each of its chunks (shared memory).  The k-th largest of the
// threads' own largest scores is a floor of the k-th best class; only chunks that reach it are looked at again (in L1 or L2),
// about k of thousands, and what reaches it in them is sorted.  Where that gives fewer than k classes or more than LP_CAND (many
// equal scores, rows masked nearly throughout, scores that are not numbers) the classes are offered to a sorted list one by
// one.  256 x 170,000 bf16, ten best: 31 us, 175 us with all offered one by one, 113 us where scores spread evenly over 8 to 16 have
// thousands of equals at the top.  Chunks
// fetched a step ahead, through shared memory or registers, other numbers of parts, or a maximum of which the sums follow only every
// e^2: 33 to 44 us; a part's results pushed to the first block instead of fetched by it: 34 us.
constexpr int LP_CAND = 256;
constexpr int LP_CHUNKS = 48;  // chunks of a thread at most: shared memory

template <typename T, int W, bool CLUSTER>
__global__ void __launch_bounds__(256)
log_probs_kernel(const LpParams P) {
    if constexpr (W == 1) pdl_wait(); else pdl_wait_exclusive();  // (blocks of the next kernel that come up early lie unevenly)
    constexpr int PER = Chunk<T>::N;
    extern __shared__ float sh_max[];  // [chunks of a thread][256]
    __shared__ LpStats sh_stats[8];
    __shared__ uint64_t sh_cand[W == 1 ? 8 : 1][LP_CAND];
    __shared__ uint64_t sh_keys[W == 1 ? 1 : 8][LP_TOP];
    __shared__ float sh_sorted[W == 1 ? 1 : 8][32], sh_floor;
    __shared__ int sh_count[8], sh_owner;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = W == 1 ? (int64_t)blockIdx.x * 8 + warp : (int64_t)blockIdx.x / P.parts;
    const int part = W == 1 ? 0 : (int)(blockIdx.x % P.parts);
    if (row >= P.N) return;  // (W = 1: a whole warp; no block-wide step follows)
    const T* const z = (const T*)P.z;
    // 16-byte chunks of the whole matrix that hold elements of the row (of the part): the row's first and last may hold others' too
    const int64_t e0 = row * P.C, all = P.N * P.C;
    int64_t c0 = e0 / PER, c1 = (e0 + P.C + PER - 1) / PER;
    if (P.parts > 1) {
        const int64_t per = (c1 - c0 + P.parts - 1) / P.parts, n0 = c0 + part * per, n1 = n0 + per;
        c1 = n1 < c1 ? n1 : c1;
        c0 = n0;
    }
    const int count = c1 > c0 ? (int)(c1 - c0) : 0;
    const T* const zc = z + c0 * PER;
    const int first_class = (int)(c0 * PER - e0);             // class of the first element of chunk 0; negative: another row's
    const int whole = (int)((all - c0 * PER) / PER < count ? (all - c0 * PER) / PER : count);  // chunks that end inside the matrix
    const int me = W == 1 ? lane : threadIdx.x;
    constexpr int STEP = W * 32;
    auto load = [&](int i) {
        if (i < whole) return ld_16(zc + (int64_t)i * PER);
        union { T e[PER]; uint4 q; } x;
#pragma unroll
        for (int k = 0; k < PER; ++k) x.e[k] = c0 * PER + (int64_t)i * PER + k < all ? zc[(int64_t)i * PER + k] : T(0.f);
        return x.q;
    };
    float z_label = 0.f;  // (asked for here, not at the end, where it would be waited for)
    if (part == 0 && me == 0 && P.logp) {
        const int y = P.label[row];
        if (y >= 0 && y < P.C) z_label = (float)z[e0 + y];
    }
    auto inside = [&](int i, int k) { return (unsigned)(first_class + i * PER + k) < (unsigned)P.C; };
    auto scores = [&](int i, uint4 v, float* f) {  // those of other rows: -inf
        Chunk<T>::unpack(v, f);
        if (!inside(i, 0) || !inside(i, PER - 1)) {
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (!inside(i, k)) f[k] = -INFINITY;
        }
    };
    LpRun run;
    run.clear();
    const bool list = P.top > 0;
    constexpr int U = 4;  // chunks in flight per lane
    int n = 0;
    // chunks of the row alone: all but its two ends
    const int lo = first_class < 0 ? 1 : 0, hi = (int64_t)first_class + (int64_t)count * PER > P.C ? count - 1 : count;
    for (int c = me; c - me < count; c += U * STEP) {  // the same for all lanes
        uint4 v[U];
        if (c >= lo && c + (U - 1) * STEP < hi) {  // four whole chunks: the maximum rises once at most
            float cm[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = ld_16(zc + (int64_t)(c + u * STEP) * PER);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                cm[u] = lp_chunk_max<T>(v[u]);
                if (list) sh_max[(n + u) * 256 + threadIdx.x] = cm[u];
            }
            const float bm = fmaxf(fmaxf(cm[0], cm[1]), fmaxf(cm[2], cm[3]));
            n += U;
            if (bm > run.m) run.raise(bm);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[PER];
                Chunk<T>::unpack(v[u], f);
#pragma unroll
                for (int k = 0; k < PER; k += 2) run.add<false>(f[k], f[k + 1]);
            }
            continue;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c + u * STEP < count) v[u] = load(c + u * STEP);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c + u * STEP >= count) break;
            float f[PER];
            scores(c + u * STEP, v[u], f);
            float cm = f[0];
#pragma unroll
            for (int k = 1; k < PER; ++k) cm = fmaxf(cm, f[k]);
            if (list) sh_max[n * 256 + threadIdx.x] = cm;
            ++n;
            if (cm > run.m) run.raise(cm);
#pragma unroll
            for (int k = 0; k < PER; k += 2) run.add<false>(f[k], f[k + 1]);
        }
    }
    const float mine = run.m;  // its own largest score
    LpStats st = run.stats();
    lp_join_lanes(st, lane);
    if constexpr (W > 1) {
        if (lane == 0) sh_stats[warp] = st;
        __syncthreads();
        st = lp_join_warps(sh_stats, lane);
    }
    if (fabsf(st.m) > LpRun::FAR && fabsf(st.m) < INFINITY) {  // far from zero: once more, by exact differences
        run.from_maximum(mine);
        for (int c = me; c < count; c += STEP) {
            float f[PER];
            scores(c, load(c), f);
#pragma unroll
            for (int k = 0; k < PER; k += 2) run.add<true>(f[k], f[k + 1]);
        }
        st = run.stats();
        lp_join_lanes(st, lane);
        if constexpr (W > 1) {
            __syncthreads();  // the first sums have been read
            if (lane == 0) sh_stats[warp] = st;
            __syncthreads();
            st = lp_join_warps(sh_stats, lane);
        }
    }
    // One class takes most of it: the sum beside its own 1 has lost digits in the thread that holds it.  That thread's chunks again,
    // without the 1, by its warp; the other threads' sums stand.
    if (st.s < 0.0625f && st.m > -INFINITY && st.m < INFINITY) {
        const uint32_t at = __ballot_sync(0xFFFFFFFFu, mine == st.m);
        int owner = at ? warp * 32 + __ffs(at) - 1 : 256;
        if constexpr (W > 1) {
            if (threadIdx.x == 0) sh_owner = 256;
            __syncthreads();
            if (lane == 0) atomicMin(&sh_owner, owner);
            __syncthreads();
            owner = sh_owner;
        }
        LpStats own = run.stats();
        if (owner / 32 == warp) {
            const int who = W == 1 ? owner % 32 : owner;
            LpStats again;
            again.clear();
            again.m = st.m;
            bool taken = false;  // the first of its classes at the maximum
            for (int c = who; c < count; c += 32 * STEP) {
                const int i = c + lane * STEP;
                float f[PER];
                bool hit = false;
                if (i < count) {
                    scores(i, load(i), f);
#pragma unroll
                    for (int k = 0; k < PER; ++k) hit |= f[k] == st.m;
                }
                const uint32_t hits = __ballot_sync(0xFFFFFFFFu, hit);
                bool skip = !taken && hits && lane == __ffs(hits) - 1;
                taken |= hits != 0;
                if (i < count) {
#pragma unroll
                    for (int k = 0; k < PER; ++k) {
                        if (skip && f[k] == st.m) skip = false;
                        else again.add(f[k], st.m);
                    }
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                again.s += __shfl_xor_sync(0xFFFFFFFFu, again.s, o);
                again.t += __shfl_xor_sync(0xFFFFFFFFu, again.t, o);
            }
            if (lane == owner % 32) own = again;
        }
        st = own;
        lp_join_lanes(st, lane);
        if constexpr (W > 1) {
            if (lane == 0) sh_stats[warp] = st;
            __syncthreads();
            st = lp_join_warps(sh_stats, lane);
        }
    }
    uint64_t best = 0;
    if (list) {
        float floor = mine;
        const int g = W == 1 ? warp : 0;
        if (lane == 0) sh_count[warp] = 0;
        if constexpr (W == 1) {
            floor = __shfl_sync(0xFFFFFFFFu, lp_sort(floor, lane), P.top - 1);
            __syncwarp();
        } else if (P.top <= 16) {  // the k-th largest of 32 groups of eight threads will do: half as many groups more reach it, by chance, than classes are listed
            sh_sorted[warp][lane] = mine;
            __syncthreads();
            for (int w = 0; w < W; ++w) floor = fmaxf(floor, sh_sorted[w][lane]);
            floor = __shfl_sync(0xFFFFFFFFu, lp_sort(floor, lane), P.top - 1);
        } else {
            floor = lp_sort(floor, lane);
            sh_sorted[warp][lane] = floor;
            __syncthreads();
            if (warp == 0) {
                for (int w = 1; w < W; ++w) floor = lp_merge(floor, sh_sorted[w][lane], lane);
                if (lane == P.top - 1) sh_floor = floor;
            }
            __syncthreads();
            floor = sh_floor;
        }
        for (int k = 0; k < n && mine >= floor; ++k) {
            if (!(sh_max[k * 256 + threadIdx.x] >= floor)) continue;
            const int i = k * STEP + me;
            float f[PER];
            Chunk<T>::unpack(load(i), f);
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (f[e] >= floor && inside(i, e)) {
                    const int at = atomicAdd(&sh_count[g], 1);
                    if (at < LP_CAND) sh_cand[g][at] = lp_key(f[e], (uint32_t)(first_class + i * PER + e));
                }
        }
        if constexpr (W == 1) __syncwarp(); else __syncthreads();
        const int found = sh_count[g];
        if (found >= P.top && found <= LP_CAND) {
            if (W == 1 || warp == 0) best = lp_best_of(sh_cand[g], found, lane);
        } else {
            LpTop one;
            one.clear();
            for (int c = 0; c < count; c += STEP) {
                const int i = c + me;
                float f[PER];
                if (i < count) Chunk<T>::unpack(load(i), f);
#pragma unroll
                for (int e = 0; e < PER; ++e) one.offer(i < count && inside(i, e) ? lp_key(f[e], (uint32_t)(first_class + i * PER + e)) : 0, P.top, lane);
            }
            best = one.key;
            if constexpr (W > 1) {
                sh_keys[warp][lane] = best;
                __syncthreads();
                if (warp == 0)
                    for (int w = 1; w < W; ++w) best = lp_merge(best, sh_keys[w][lane], lane);
            }
        }
    }
    if constexpr (CLUSTER) {  // the parts of a row are the blocks of a cluster: the first one joins them
        namespace cg = cooperative_groups;
        cg::cluster_group all_parts = cg::this_cluster();
        __shared__ LpStats sh_part;  // (not sh_stats, which other warps may still read)
        __shared__ uint64_t sh_part_keys[LP_TOP];
        if (warp == 0) {
            if (lane == 0) sh_part = st;
            sh_part_keys[lane] = best;
        }
        all_parts.sync();
        if (part == 0 && warp == 0) {
            st.clear();
            if (lane < P.parts) st = *all_parts.map_shared_rank(&sh_part, lane);
            lp_join_lanes(st, lane);
            if (list)
                for (int p = 1; p < P.parts; ++p) best = lp_merge(best, *all_parts.map_shared_rank(&sh_part_keys[lane], p), lane);
        }
        all_parts.sync();  // nobody leaves while it is read
        if (part != 0 || warp != 0) return;
    } else if constexpr (W > 1) {
        if (warp != 0) return;
        if (P.parts > 1) {
            const int64_t at = row * P.parts + part;
            if (lane == 0) { P.stats[at * 4] = st.m; P.stats[at * 4 + 1] = st.s; P.stats[at * 4 + 2] = st.t; }
            if (lane < P.top) P.keys[at * P.top + lane] = best;
            return;
        }
    }
    lp_finish<T>(P, row, st, z_label, best, lane);
}

// The parts of a row joined: a block per row.  Only parts whose best class is among the k best such can hold one of the k best.
template <typename T>
__global__ void __launch_bounds__(256)
log_probs_join_kernel(const LpParams P) {
    pdl_wait();
    __shared__ LpStats sh_stats[8];
    __shared__ uint64_t sh_keys[8][32], sh_cand[LP_TOP * LP_TOP], sh_floor;
    __shared__ int sh_count;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = blockIdx.x, first = row * P.parts;
    LpStats st;
    st.clear();
    uint64_t top = 0;  // of this warp's parts, their best classes
    for (int p0 = warp * 32; p0 < P.parts; p0 += 256) {
        const int p = p0 + lane;
        uint64_t k = 0;
        if (p < P.parts) {
            const float4 v = *reinterpret_cast<const float4*>(P.stats + (first + p) * 4);
            LpStats q;
            q.m = v.x; q.s = v.y; q.t = v.z;
            st.join(q);
            if (P.top > 0) k = P.keys[(first + p) * P.top];
        }
        if (P.top > 0) top = lp_merge(top, lp_sort(k, lane), lane);
    }
    lp_join_lanes(st, lane);
    if (lane == 0) sh_stats[warp] = st;
    sh_keys[warp][lane] = top;
    if (threadIdx.x == 0) sh_count = 0;
    __syncthreads();
    if (P.top > 0) {
        if (warp == 0) {
            for (int w = 1; w < 8; ++w) top = lp_merge(top, sh_keys[w][lane], lane);
            if (lane == P.top - 1) sh_floor = top;  // 0 where there are fewer parts than that: all of them count
        }
        __syncthreads();
        const uint64_t floor = sh_floor;
        // keys differ, so that at most `top` parts pass, with `top` keys each: they fit
        const int parts = P.parts;
        if (floor > 0) {
            for (int p = threadIdx.x; p < parts; p += 256)
                for (int j = 0; j < P.top; ++j) {
                    const uint64_t k = P.keys[(first + p) * P.top + j];
                    if (k < floor) break;
                    sh_cand[atomicAdd(&sh_count, 1)] = k;
                }
        } else {
            for (int64_t i = threadIdx.x; i < (int64_t)parts * P.top; i += 256) {
                const uint64_t k = P.keys[first * P.top + i];
                if (k) sh_cand[atomicAdd(&sh_count, 1)] = k;  // fewer than `top` parts have any
            }
        }
        __syncthreads();
    }
    if (warp != 0) return;
    st = lp_join_warps(sh_stats, lane);
    lp_finish<T>(P, row, st, lane == 0 && P.logp && (unsigned)P.label[row] < (unsigned)P.C ? (float)((const T*)P.z)[row * P.C + P.label[row]] : 0.f, P.top > 0 ? lp_best_of(sh_cand, sh_count, lane) : 0, lane);
}

struct LpGradParams {
    const void* z;
    const int32_t* label;
    int64_t N;
    int C;
    const float *lse, *lse_rest, *entropy, *dlogp, *dentropy;  // entropy and dentropy together, or neither; dlogp may be nullptr
    void* dz;
};

// What a row's gradient needs; none: nothing to choose from, so that nothing depends on the scores.
// REST: with what the rounding of lse left out.  z - lse is then off by its own rounding alone, not by half a unit of lse's last bit (of the row's
// every p: 5e-4 at lse = 1e4, all of it from about 1e7 on), and a nearly sure label's 1 - p keeps its digits.
// 2048 x 50,000 bf16 74 us, 170,000 x 47 fp32 27 us (without: 67 and 21); 20,000 x 2000 fp32 76 us (85).
template <bool REST>
struct LpRow {
    float lse, H, g, h;  // (REST: H less the rest, so that z - lse serves in both places, and the rest's share of the exponent)
    float rest, shift;
    int y;
    bool none;
    __device__ __forceinline__ void read(const LpGradParams& P, int64_t row) {
        lse = P.lse[row];
        none = lse < -1e30f;
        y = P.label ? P.label[row] : -1;
        g = P.dlogp && y >= 0 && y < P.C && !none ? P.dlogp[row] : 0.f;
        h = P.dentropy ? P.dentropy[row] : 0.f;
        H = P.dentropy ? P.entropy[row] : 0.f;
        if constexpr (REST) {
            rest = P.lse_rest[row];
            shift = rest * -1.4426950408889634f;
            H -= rest;
        }
    }
    // without the label's own share.  A class at -inf: p = 0 times what is finite for all h up to 1e36 (p is 0 from log p = -88 on, so
    // that the bound changes no other; a comparison of p instead: 2048 x 50,000 bf16 67 -> 71 us)
    __device__ __forceinline__ float operator()(float z) const {
        const float lp = z - lse;
        return none ? 0.f : -p(lp) * fmaf(h, fmaxf(lp, -128.f) + H, g);
    }
    // (REST) the label, its share g (1 - p) included
    __device__ __forceinline__ float at_label(float z) const {
        const float lp = z - lse;
        return none ? 0.f : -p(lp) * h * (fmaxf(lp, -128.f) + H) - expm1f(lp - rest) * g;
    }
    __device__ __forceinline__ float p(float lp) const { return REST ? LpRun::exp2_(fmaf(lp, 1.4426950408889634f, shift)) : lp_exp(lp); }
};

// element k of a chunk
template <typename T>
__device__ __forceinline__ float lp_pick(uint4 v, int k) {
    float f[Chunk<T>::N], x = 0.f;
    Chunk<T>::unpack(v, f);
#pragma unroll
    for (int q = 0; q < Chunk<T>::N; ++q) x = q == k ? f[q] : x;
    return x;
}

// Long rows, from LG_CLASSES on: a block takes LG_CHUNKS chunks of 16 bytes of one row.  Chunks that two rows share are written by both, element
// by element.  2048 x 50,000 bf16 67 us (6.1 TB/s).  This kernel / the one below, which divides to find a chunk's row, 20,000 rows: 349 classes fp32
// 31 / 13 us, bf16 36 / 11; 1000 classes 42 / 46, 36 / 26; 2000 classes 58 / 86, 47 / 59; 4000 classes 95 / 160, 64 / 110.  (fp32 would gain from
// a border of 1000.)
constexpr int LG_CLASSES = 2048;
constexpr int LG_PER = 4, LG_CHUNKS = 256 * LG_PER;

template <typename T, bool REST>
__global__ void __launch_bounds__(256)
log_probs_backward_rows_kernel(const LpGradParams P, int parts) {
    pdl_wait();
    constexpr int PER = Chunk<T>::N;
    const int64_t row = blockIdx.x / parts, all = P.N * P.C;
    const int64_t e0 = row * P.C, e1 = e0 + P.C, c1 = (e1 + PER - 1) / PER;
    const int64_t c0 = e0 / PER + (int64_t)(blockIdx.x % parts) * LG_CHUNKS + threadIdx.x;
    const T* const z = (const T*)P.z;
    T* const dz = (T*)P.dz;
    LpRow<REST> R;
    R.read(P, row);
    const int64_t hit = R.y >= 0 && R.y < P.C ? e0 + R.y : -1;
    uint4 v[LG_PER];
#pragma unroll
    for (int u = 0; u < LG_PER; ++u) {
        const int64_t i = c0 + u * 256;
        if (i < c1 && (i + 1) * PER <= all) v[u] = ld_16(z + i * PER);
    }
    float share = R.g;
    if constexpr (REST) {  // by the thread that writes the label
        const int64_t q = hit / PER - c0;
        if (hit >= 0 && q >= 0 && q < LG_CHUNKS && q % 256 == 0) share = R.at_label((float)z[hit]);
    }
#pragma unroll
    for (int u = 0; u < LG_PER; ++u) {
        const int64_t i = c0 + u * 256;
        if (i >= c1) break;
        if (i * PER >= e0 && (i + 1) * PER <= e1) {
            float f[PER];
            Chunk<T>::unpack(v[u], f);
#pragma unroll
            for (int k = 0; k < PER; ++k) f[k] = R(f[k]);
            if (hit >= i * PER && hit < (i + 1) * PER) {
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (hit == i * PER + k) f[k] = REST ? share : f[k] + share;
            }
            *reinterpret_cast<uint4*>(dz + i * PER) = Chunk<T>::pack(f);
        } else {
            for (int k = 0; k < PER; ++k) {
                const int64_t e = i * PER + k;
                if (e >= e0 && e < e1) dz[e] = T(REST && e == hit ? share : R((float)z[e]) + (e == hit ? share : 0.f));
            }
        }
    }
}

// short rows: a chunk of 16 bytes per thread and step, whatever rows its elements lie in
template <typename T, typename I, bool REST>
__global__ void __launch_bounds__(256)
log_probs_backward_kernel(const LpGradParams P) {
    pdl_wait();
    constexpr int PER = Chunk<T>::N;
    const int64_t all = P.N * P.C, chunks = (all + PER - 1) / PER;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
        const bool whole = (i + 1) * PER <= all;
        float f[PER];
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (whole) {
            raw = ld_16((const T*)P.z + i * PER);
            Chunk<T>::unpack(raw, f);
        } else {
#pragma unroll
            for (int k = 0; k < PER; ++k) f[k] = i * PER + k < all ? (float)((const T*)P.z)[i * PER + k] : 0.f;
            if constexpr (REST) raw = Chunk<T>::pack(f);  // (exact)
        }
        int64_t row = (I)(i * PER) / (I)P.C;
        int c = (int)(i * PER - row * P.C);
        LpRow<REST> R;
        R.read(P, row);
        uint32_t labels = 0;  // (REST: expm1 once per label, not once per element: 170k x 47 fp32 29 -> 27 us)
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if constexpr (REST) {
                f[k] = R(f[k]);
                if (c == R.y) labels |= 1u << k;
            } else {
                f[k] = R(f[k]) + (c == R.y ? R.g : 0.f);
            }
            if (++c == P.C) {
                c = 0;
                if (++row < P.N && k + 1 < PER) R.read(P, row);
            }
        }
        if constexpr (REST) {
            while (labels) {
                const int at = __ffs(labels) - 1;
                labels &= labels - 1;
                R.read(P, (I)(i * PER + at) / (I)P.C);
                const float v = R.at_label(lp_pick<T>(raw, at));
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (k == at) f[k] = v;
            }
        }
        if (whole) *reinterpret_cast<uint4*>((T*)P.dz + i * PER) = Chunk<T>::pack(f);
        else
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (i * PER + k < all) ((T*)P.dz)[i * PER + k] = T(f[k]);
    }
}

// Blocks per row: what makes the fewest rounds of four blocks per SM times the chunks per thread of a block, to which its fixed part
// (joining, sorting) adds about 14; a block has 8 KB of the row at least, a thread LP_CHUNKS chunks at most.
static int64_t lp_parts(int64_t N, int64_t C, int s) {
    const int64_t bytes = C * s, least = ceil_div(bytes + 16, (int64_t)LP_CHUNKS * 256 * 16 - 16);
    int64_t most = bytes / (8 * 1024);
    if (most > 592) most = 592;
    if (N >= 592 * 8 || most <= least) return least;
    auto cost = [&](int64_t p) { return (double)ceil_div(N * p, 592) * ((double)bytes / 4096 / (double)p + 14.0); };
    int64_t best = least;
    for (int64_t p = least + 1; p <= most; ++p)
        if (cost(p) < 0.98 * cost(best)) best = p;
    return best;
}

// A thread per row: few classes, and rows enough to fill the SMs with threads.  By a thread / by a warp, fp32, five best: 170,000 x 47 12.3 / 158 us, 16,384 x 64
// 7.3 / 17.0, 4096 x 64 6.1 / 6.0, 2048 x 64 6.0 / 5.5, 256 x 64 5.9 / 4.1.  (Up to 16 classes a thread is the faster one from 256 rows on: 3.6 / 4.2.)
static bool lp_few(int64_t N, int C) { return C <= LP_FEW && N >= 4096; }

// launch_overlapped with clusters
template <class... Params, class... Args>
static void launch_cluster(void (*kernel)(Params...), unsigned blocks, unsigned size, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = size;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);  // errors: GNN_CHECK_LAUNCH of the caller
}

struct LpWs {
    int64_t parts;
    size_t keys, bytes;
    LpWs(int64_t N, int C, int top, gnn_dtype dtype) {
        parts = N > 0 && C > LP_WARP_CLASSES ? lp_parts(N, C, elem_size(dtype)) : 1;
        keys = parts > LP_CLUSTER ? up256((size_t)N * parts * 16) : 0;
        bytes = keys + (parts > LP_CLUSTER ? up256((size_t)N * parts * top * 8) : 0);
    }
};

}  // namespace gnn

using namespace gnn;

extern "C" {

size_t gnn_log_probs_workspace(int32_t N, int C, int top, gnn_dtype dtype) {
    if (N < 0 || C <= 0 || top < 0 || top > LP_TOP || (dtype != GNN_F32 && dtype != GNN_BF16)) return 0;
    return LpWs(N, C, top, dtype).bytes;
}

gnn_status gnn_log_probs(const void* Z, const int32_t* label, int32_t N, int C, gnn_dtype dtype, int top, float* logp, float* entropy, float* lse,
                         float* top_logp, int32_t* top_idx, void* ws, size_t ws_bytes, gnn_stream stream) {
    return gnn_log_probs_rest(Z, label, N, C, dtype, top, logp, entropy, lse, nullptr, top_logp, top_idx, ws, ws_bytes, stream);
}

gnn_status gnn_log_probs_rest(const void* Z, const int32_t* label, int32_t N, int C, gnn_dtype dtype, int top, float* logp, float* entropy, float* lse,
                              float* lse_rest, float* top_logp, int32_t* top_idx, void* ws, size_t ws_bytes, gnn_stream stream) {
    const char* who = "gnn_log_probs";
    GNN_REQUIRE(N >= 0 && C > 0, GNN_ERR_INVALID_ARG, "%s: bad shape", who);
    GNN_REQUIRE(dtype == GNN_F32 || dtype == GNN_BF16, GNN_ERR_INVALID_ARG, "%s: bad dtype", who);
    GNN_REQUIRE(top >= 0 && top <= C, GNN_ERR_INVALID_ARG, "%s: top is %d of %d classes", who, top, C);
    GNN_REQUIRE(top <= LP_TOP, GNN_ERR_UNSUPPORTED, "%s: top up to %d", who, LP_TOP);
    GNN_REQUIRE(!logp || label || N == 0, GNN_ERR_INVALID_ARG, "%s: logp needs label", who);
    if (N == 0) return GNN_OK;
    GNN_REQUIRE(Z && (top == 0 || (top_logp && top_idx)), GNN_ERR_INVALID_ARG, "%s: null argument", who);
    GNN_REQUIRE(aligned16(Z), GNN_ERR_INVALID_ARG, "%s: Z must be 16-byte aligned", who);
    const LpWs lw(N, C, top, dtype);
    GNN_REQUIRE(lw.bytes == 0 || (ws && ws_bytes >= lw.bytes && aligned16(ws)), GNN_ERR_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes needed, 16-byte aligned", who, lw.bytes);
    cudaStream_t st = as_stream(stream);
    LpParams P;
    P.z = Z; P.label = label; P.N = N; P.C = C; P.top = top;
    P.logp = logp; P.entropy = entropy; P.lse = lse; P.lse_rest = lse_rest; P.top_logp = top_logp; P.top_idx = top_idx;
    P.parts = (int)lw.parts; P.stats = (float*)ws; P.keys = (uint64_t*)((char*)ws + lw.keys);
    const bool f32 = dtype == GNN_F32;
    const int64_t chunks = (int64_t)C / (f32 ? 4 : 8) + 2;  // of a row, both ends cut
    if (lp_few(N, C)) {
        const dim3 grid((unsigned)ceil_div(N, LP_ROWS));
        const size_t smem = ((size_t)LP_ROWS * lp_few_stride(C) + 8) * 4;
        auto run = [&](auto kernel) { launch_overlapped(kernel, grid, dim3(LP_ROWS), smem, st, P); };
        if (f32) C <= 16 ? run(log_probs_few_kernel<float, 2>) : C <= 32 ? run(log_probs_few_kernel<float, 4>) : C <= 48 ? run(log_probs_few_kernel<float, 6>) : run(log_probs_few_kernel<float, 8>);
        else C <= 16 ? run(log_probs_few_kernel<__nv_bfloat16, 2>) : C <= 32 ? run(log_probs_few_kernel<__nv_bfloat16, 4>) : C <= 48 ? run(log_probs_few_kernel<__nv_bfloat16, 6>) : run(log_probs_few_kernel<__nv_bfloat16, 8>);
    } else if (C <= LP_WARP_CLASSES) {
        const dim3 grid((unsigned)ceil_div(N, 8));
        const size_t smem = top > 0 ? (size_t)ceil_div(chunks, 32) * 1024 : 0;
        if (f32) launch_overlapped(log_probs_kernel<float, 1, false>, grid, dim3(256), smem, st, P);
        else launch_overlapped(log_probs_kernel<__nv_bfloat16, 1, false>, grid, dim3(256), smem, st, P);
    } else {
        const int64_t blocks = (int64_t)N * lw.parts;
        GNN_REQUIRE(blocks <= INT32_MAX, GNN_ERR_UNSUPPORTED, "%s: too many rows", who);
        const size_t smem = top > 0 ? (size_t)ceil_div(ceil_div(chunks, lw.parts), 256) * 1024 : 0;
        const bool cluster = lw.parts > 1 && lw.parts <= LP_CLUSTER;
        auto run = [&](auto kernel, int slot) {
            const gnn_status rc = allow_big_smem(who, (const void*)kernel, slot, LP_CHUNKS * 1024);
            if (rc != GNN_OK) return rc;
            if (cluster) launch_cluster(kernel, (unsigned)blocks, (unsigned)lw.parts, smem, st, P);
            else launch_overlapped(kernel, dim3((unsigned)blocks), dim3(256), smem, st, P);
            return GNN_OK;
        };
        const gnn_status rc = f32 ? cluster ? run(log_probs_kernel<float, 8, true>, LP_SLOT) : run(log_probs_kernel<float, 8, false>, LP_SLOT + 1)
                                  : cluster ? run(log_probs_kernel<__nv_bfloat16, 8, true>, LP_SLOT + 2) : run(log_probs_kernel<__nv_bfloat16, 8, false>, LP_SLOT + 3);
        if (rc != GNN_OK) return rc;
        if (lw.parts > LP_CLUSTER) {
            const dim3 grid((unsigned)N);
            if (f32) launch_overlapped(log_probs_join_kernel<float>, grid, dim3(256), 0, st, P);
            else launch_overlapped(log_probs_join_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, P);
        }
    }
    GNN_CHECK_LAUNCH(who);
    return GNN_OK;
}

gnn_status gnn_log_probs_backward(const void* Z, const int32_t* label, const float* lse, const float* entropy, const float* dlogp, const float* dentropy,
                                  int32_t N, int C, gnn_dtype dtype, void* dZ, gnn_stream stream) {
    return gnn_log_probs_rest_backward(Z, label, lse, nullptr, entropy, dlogp, dentropy, N, C, dtype, dZ, stream);
}

gnn_status gnn_log_probs_rest_backward(const void* Z, const int32_t* label, const float* lse, const float* lse_rest, const float* entropy, const float* dlogp,
                                       const float* dentropy, int32_t N, int C, gnn_dtype dtype, void* dZ, gnn_stream stream) {
    const char* who = "gnn_log_probs_backward";
    GNN_REQUIRE(N >= 0 && C > 0, GNN_ERR_INVALID_ARG, "%s: bad shape", who);
    GNN_REQUIRE(dtype == GNN_F32 || dtype == GNN_BF16, GNN_ERR_INVALID_ARG, "%s: bad dtype", who);
    GNN_REQUIRE(!dlogp || label || N == 0, GNN_ERR_INVALID_ARG, "%s: dlogp needs label", who);
    GNN_REQUIRE(!dentropy || entropy || N == 0, GNN_ERR_INVALID_ARG, "%s: dentropy needs entropy", who);
    if (N == 0) return GNN_OK;
    GNN_REQUIRE(Z && lse && dZ, GNN_ERR_INVALID_ARG, "%s: null argument", who);
    GNN_REQUIRE(aligned16(Z) && aligned16(dZ), GNN_ERR_INVALID_ARG, "%s: matrices must be 16-byte aligned", who);
    cudaStream_t st = as_stream(stream);
    LpGradParams P;
    P.z = Z; P.label = label; P.N = N; P.C = C; P.lse = lse; P.lse_rest = lse_rest; P.entropy = entropy; P.dlogp = dlogp; P.dentropy = dentropy; P.dz = dZ;
    const int per = dtype == GNN_F32 ? 4 : 8;
    const int64_t parts = ceil_div((int64_t)C / per + 2, LG_CHUNKS), blocks = parts * N;
    const bool narrow = (int64_t)N * C + 8 <= UINT32_MAX;  // the division that finds a chunk's row
    auto run = [&](auto t, auto rest) {
        using T = decltype(t);
        constexpr bool REST = decltype(rest)::value;
        if (C >= LG_CLASSES && blocks <= INT32_MAX) {
            launch_overlapped(log_probs_backward_rows_kernel<T, REST>, dim3((unsigned)blocks), dim3(256), 0, st, P, (int)parts);
            return;
        }
        const dim3 grid((unsigned)grid_for(ceil_div((int64_t)N * C, per), 256));
        if (narrow) launch_overlapped(log_probs_backward_kernel<T, uint32_t, REST>, grid, dim3(256), 0, st, P);
        else launch_overlapped(log_probs_backward_kernel<T, int64_t, REST>, grid, dim3(256), 0, st, P);
    };
    if (dtype == GNN_F32) lse_rest ? run(float(), std::true_type()) : run(float(), std::false_type());
    else lse_rest ? run(__nv_bfloat16(), std::true_type()) : run(__nv_bfloat16(), std::false_type());
    GNN_CHECK_LAUNCH(who);
    return GNN_OK;
}

}  // extern "C"
