// What follows the last layer of a node classifier or of an entity ranker: per row of scores z [N,C]
//   lse = log sum_c exp z_c,  logp = z_label - lse,  H = -sum_c p_c log p_c (p = exp(z - lse)),  the k best classes and their log p
// in one pass over the scores, and the gradient of logp and H
//   dz_c = dlogp ([c = label] - p_c) - dH p_c (log p_c + H).
//
// Running statistics of a part of a row: m (largest score), s = sum of exp(z - m) over all classes BUT one of those at m, and
// t = sum of exp(z - m) (z - m).  Then lse = m + log1p(s) and H = log1p(s) - t / (1 + s): without the leading 1 in the sum, a
// row whose best class is nearly sure keeps the digits of its small log p and entropy.  Two parts are joined by scaling the one
// with the smaller maximum, whose own maximum counts again: exp(m1 - m2) (s1 + 1).
// The k best: keys of (score, lower index first) that are all different, sorted over the lanes of a warp; a chunk whose largest
// score does not pass the worst of them is left alone.
#include "common.cuh"

namespace gnn {

constexpr int LP_TOP = 32;  // classes listed at most: a lane each

__device__ __forceinline__ float lp_exp(float d) {  // exp of d <= 0: 2^(d log2 e); the error of the product reaches what is below e^-10 by 1e-6 of it
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(d * 1.4426950408889634f));
    return e;
}

struct LpStats {
    float m, s, t;
    __device__ __forceinline__ void clear() { m = -INFINITY; s = 0.f; t = 0.f; }
    // the maximum becomes v > m
    __device__ __forceinline__ void raise(float v) {
        const float d = m - v, f = lp_exp(d), c = f * (s + 1.f);  // m = -inf: f = 0
        t = fmaf(fmaxf(d, -1000.f), c, f * t);
        s = c;
        m = v;
    }
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
        t += fmaf(d, c, f * o.t);
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

struct LpParams {
    const void* z;
    const int32_t* label;  // or nullptr
    int64_t N;
    int C, top;
    float *logp, *entropy, *lse, *top_logp;  // each may be nullptr
    int32_t* top_idx;
    int parts;          // blocks per row (whole-block rows)
    float* stats;       // [N][parts][4] where parts > 1
    uint64_t* keys;     // [N][parts][top]
};

// what a row answers, from its statistics (all lanes) and its best (a lane each)
template <typename T>
__device__ __forceinline__ void lp_finish(const LpParams& P, int64_t row, const LpStats& st, const LpTop& best, int lane) {
    const float nan = __uint_as_float(0x7FC00000u);
    const bool bad = st.s != st.s || st.m == INFINITY, none = st.m == -INFINITY;
    const float tail = log1pf(st.s);
    const float lse = bad ? nan : none ? -INFINITY : st.m + tail;
    // z - lse as (z - m) - log1p(s): exact where z is the largest
    auto logp = [&](float z) { return bad ? nan : none || z == -INFINITY ? -INFINITY : (z - st.m) - tail; };
    if (lane == 0) {
        if (P.lse) P.lse[row] = lse;
        if (P.entropy) P.entropy[row] = bad ? nan : none ? 0.f : tail - st.t / (1.f + st.s);
        if (P.logp) {
            const int y = P.label[row];
            P.logp[row] = y >= 0 && y < P.C ? logp((float)((const T*)P.z)[row * P.C + y]) : 0.f;
        }
    }
    if (lane < P.top) {
        P.top_idx[row * P.top + lane] = (int32_t)lp_class(best.key);
        P.top_logp[row * P.top + lane] = logp(lp_score(best.key));
    }
}

// rows by W warps (1: eight rows a block; 8: a row, or a part of one, per block)
template <typename T, int W>
__global__ void __launch_bounds__(256)
log_probs_kernel(const LpParams P) {
    pdl_wait();
    constexpr int PER = Chunk<T>::N;
    __shared__ LpStats sh_stats[8];
    __shared__ uint64_t sh_keys[8][LP_TOP];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = W == 1 ? (int64_t)blockIdx.x * 8 + warp : (int64_t)blockIdx.x / P.parts;
    const int part = W == 1 ? 0 : (int)(blockIdx.x % P.parts);
    if (row >= P.N) return;  // (W = 1: a whole warp; no block-wide step follows)
    const T* const z = (const T*)P.z;
    // 16-byte chunks of the whole matrix that hold elements of the row: the first and the last may hold others' too
    const int64_t e0 = row * P.C, e1 = e0 + P.C, all = P.N * P.C;
    int64_t c0 = e0 / PER, c1 = (e1 + PER - 1) / PER;
    if (P.parts > 1) {
        const int64_t per = (c1 - c0 + P.parts - 1) / P.parts, n0 = c0 + part * per, n1 = n0 + per;
        c1 = n1 < c1 ? n1 : c1;
        c0 = n0;
    }
    LpStats st;
    LpTop best;
    st.clear();
    best.clear();
    constexpr int U = 4;  // chunks in flight per lane
    const int me = W == 1 ? lane : threadIdx.x;
    constexpr int STEP = W * 32;
    for (int64_t c = c0; c < c1; c += U * STEP) {  // the same for all lanes
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = c + u * STEP + me;
            if (i < c1) {
                if ((i + 1) * PER <= all) v[u] = ld_16(z + i * PER);
                else {
                    union { T e[PER]; uint4 q; } x;
#pragma unroll
                    for (int k = 0; k < PER; ++k) x.e[k] = i * PER + k < all ? z[i * PER + k] : T(0.f);
                    v[u] = x.q;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c + u * STEP >= c1) break;  // uniform
            const int64_t i = c + u * STEP + me;
            float f[PER];
            Chunk<T>::unpack(v[u], f);
            const bool on = i < c1;
            const bool edge = !on || i * PER < e0 || (i + 1) * PER > e1;
            bool in[PER];
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                in[k] = !edge || (on && i * PER + k >= e0 && i * PER + k < e1);
                if (!in[k]) f[k] = -INFINITY;
            }
            float cm = f[0];
#pragma unroll
            for (int k = 1; k < PER; ++k) cm = fmaxf(cm, f[k]);
            if (cm > st.m) {
                st.raise(cm);
                bool taken = false;
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    const bool skip = !taken && f[k] == cm;
                    taken |= skip;
                    if (!skip) st.add(f[k], cm);
                }
            } else {
                const float base = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
                for (int k = 0; k < PER; ++k) st.add(f[k], base);
            }
            if (P.top > 0) {
                // a class in an earlier chunk wins a tie: only a larger score passes, once the list is full
                const bool passes = (best.last >> 32) <= 1u ? on : cm > lp_score(best.last);
                if (__any_sync(0xFFFFFFFFu, passes)) {
#pragma unroll
                    for (int k = 0; k < PER; ++k) best.offer(passes && in[k] ? lp_key(f[k], (uint32_t)(i * PER + k - e0)) : 0, P.top, lane);
                }
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        LpStats q;
        q.m = __shfl_xor_sync(0xFFFFFFFFu, st.m, o);
        q.s = __shfl_xor_sync(0xFFFFFFFFu, st.s, o);
        q.t = __shfl_xor_sync(0xFFFFFFFFu, st.t, o);
        // both sides of a pair join in the same order
        if (lane & o) { LpStats a = q; a.join(st); st = a; } else st.join(q);
    }
    if constexpr (W > 1) {
        if (lane == 0) sh_stats[warp] = st;
        sh_keys[warp][lane] = best.key;
        __syncthreads();
        if (warp != 0) return;
        for (int w = 1; w < W; ++w) {
            st.join(sh_stats[w]);
            if (P.top > 0) best.offer(lane < P.top ? sh_keys[w][lane] : 0, P.top, lane);
        }
        if (P.parts > 1) {
            const int64_t at = row * P.parts + part;
            if (lane == 0) { P.stats[at * 4] = st.m; P.stats[at * 4 + 1] = st.s; P.stats[at * 4 + 2] = st.t; }
            if (lane < P.top) P.keys[at * P.top + lane] = best.key;
            return;
        }
    }
    lp_finish<T>(P, row, st, best, lane);
}

// the parts of a row joined in ascending order: a warp per row
template <typename T>
__global__ void __launch_bounds__(256)
log_probs_join_kernel(const LpParams P) {
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= P.N) return;
    LpStats st;
    LpTop best;
    st.clear();
    best.clear();
    for (int p = 0; p < P.parts; ++p) {
        const int64_t at = row * P.parts + p;
        LpStats q;
        q.m = P.stats[at * 4]; q.s = P.stats[at * 4 + 1]; q.t = P.stats[at * 4 + 2];
        st.join(q);
        if (P.top > 0) best.offer(lane < P.top ? P.keys[at * P.top + lane] : 0, P.top, lane);
    }
    lp_finish<T>(P, row, st, best, lane);
}

struct LpGradParams {
    const void* z;
    const int32_t* label;
    int64_t N;
    int C;
    const float *lse, *entropy, *dlogp, *dentropy;  // entropy and dentropy together, or neither; dlogp may be nullptr
    void* dz;
};

// a chunk of 16 bytes per thread and step, whatever rows its elements lie in
template <typename T>
__global__ void __launch_bounds__(256)
log_probs_backward_kernel(const LpGradParams P) {
    pdl_wait();
    constexpr int PER = Chunk<T>::N;
    const int64_t all = P.N * P.C, chunks = (all + PER - 1) / PER;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
        const bool whole = (i + 1) * PER <= all;
        float f[PER];
        if (whole) Chunk<T>::unpack(ld_16((const T*)P.z + i * PER), f);
        else
#pragma unroll
            for (int k = 0; k < PER; ++k) f[k] = i * PER + k < all ? (float)((const T*)P.z)[i * PER + k] : 0.f;
        int64_t row = i * PER / P.C;
        int c = (int)(i * PER - row * P.C);
        int y = -1;
        float lse = 0.f, H = 0.f, g = 0.f, h = 0.f;
        bool fresh = true, none = false;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (row < P.N) {
                if (fresh) {
                    lse = P.lse[row];
                    y = P.label ? P.label[row] : -1;
                    g = P.dlogp && y >= 0 && y < P.C ? P.dlogp[row] : 0.f;
                    h = P.dentropy ? P.dentropy[row] : 0.f;
                    H = P.dentropy ? P.entropy[row] : 0.f;
                    none = lse < -1e30f;
                    if (none) g = 0.f;  // nothing to choose from: nothing depends on the scores
                    fresh = false;
                }
                // a class at -inf has no share, also in a row of nothing else (lse = -inf)
                float d = 0.f;
                if (f[k] != -INFINITY && !none) {
                    const float lp = f[k] - lse;
                    d = -__expf(lp) * fmaf(h, lp + H, g);
                }
                f[k] = c == y ? d + g : d;
            }
            if (++c == P.C) { c = 0; ++row; fresh = true; }
        }
        if (whole) *reinterpret_cast<uint4*>((T*)P.dz + i * PER) = Chunk<T>::pack(f);
        else
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (i * PER + k < all) ((T*)P.dz)[i * PER + k] = T(f[k]);
    }
}

// blocks per row: one, or as many as fill the SMs while each has 16 KB of the row at least
static int lp_parts(int64_t N, int64_t C, int s) {
    if (C * s < 32 * 1024 || N >= 148 * 4) return 1;
    int64_t p = (148 * 8 + N - 1) / N;
    const int64_t most = C * s / (16 * 1024);
    return (int)(p < most ? p : most > 1 ? most : 1);
}

struct LpWs {
    int parts;
    size_t keys, bytes;
    LpWs(int64_t N, int C, int top, gnn_dtype dtype) {
        parts = N > 0 ? lp_parts(N, C, elem_size(dtype)) : 1;
        keys = parts > 1 ? up256((size_t)N * parts * 16) : 0;
        bytes = keys + (parts > 1 ? up256((size_t)N * parts * top * 8) : 0);
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
    P.logp = logp; P.entropy = entropy; P.lse = lse; P.top_logp = top_logp; P.top_idx = top_idx;
    P.parts = lw.parts; P.stats = (float*)ws; P.keys = (uint64_t*)((char*)ws + lw.keys);
    const bool f32 = dtype == GNN_F32;
    if (C <= 1024) {
        const dim3 grid((unsigned)ceil_div(N, 8));
        if (f32) launch_overlapped(log_probs_kernel<float, 1>, grid, dim3(256), 0, st, P);
        else launch_overlapped(log_probs_kernel<__nv_bfloat16, 1>, grid, dim3(256), 0, st, P);
    } else {
        const int64_t blocks = (int64_t)N * lw.parts;
        GNN_REQUIRE(blocks <= INT32_MAX, GNN_ERR_UNSUPPORTED, "%s: too many rows", who);
        if (f32) launch_overlapped(log_probs_kernel<float, 8>, dim3((unsigned)blocks), dim3(256), 0, st, P);
        else launch_overlapped(log_probs_kernel<__nv_bfloat16, 8>, dim3((unsigned)blocks), dim3(256), 0, st, P);
        if (lw.parts > 1) {
            const dim3 grid((unsigned)ceil_div(N, 8));
            if (f32) launch_overlapped(log_probs_join_kernel<float>, grid, dim3(256), 0, st, P);
            else launch_overlapped(log_probs_join_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, P);
        }
    }
    GNN_CHECK_LAUNCH(who);
    return GNN_OK;
}

gnn_status gnn_log_probs_backward(const void* Z, const int32_t* label, const float* lse, const float* entropy, const float* dlogp, const float* dentropy,
                                  int32_t N, int C, gnn_dtype dtype, void* dZ, gnn_stream stream) {
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
    P.z = Z; P.label = label; P.N = N; P.C = C; P.lse = lse; P.entropy = entropy; P.dlogp = dlogp; P.dentropy = dentropy; P.dz = dZ;
    const int64_t chunks = ceil_div((int64_t)N * C, dtype == GNN_F32 ? 4 : 8);
    const dim3 grid((unsigned)grid_for(chunks, 256));
    if (dtype == GNN_F32) launch_overlapped(log_probs_backward_kernel<float>, grid, dim3(256), 0, st, P);
    else launch_overlapped(log_probs_backward_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, P);
    GNN_CHECK_LAUNCH(who);
    return GNN_OK;
}

}  // extern "C"
