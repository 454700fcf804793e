// One pipelined tensor-core kernel for products whose operand changes along the rows (segments = node types, relations), and for
// the 8-bit product, which is the same pipeline with one segment.
//
//   SG_Y   Y[i,:]  = X[i,:] * W[g(i)]           W [G,K,M]: the contraction runs down its rows, columns contiguous
//   SG_DX  dX[i,:] = dY[i,:] * W[g(i)]^T        the contraction runs along its rows
//   SG_DW  dW[g]   = X_g^T * dY_g               contraction over the rows of a segment
//   SG_I8  Y[i,m]  = sx[i] sw[m] <xq[i,:], wq[m,:]>   8-bit integers, sums in int32
//
// Rows of segment g are seg_ptr[g] .. seg_ptr[g+1]-1, known on the device only: no size is read back.
//
// Tiles of SG_Y, SG_DX and SG_I8: 128 rows of ONE segment x bn output columns.  A tile's number leads to its segment without a
// prefix sum: floor(seg_ptr[g] / 128) + g is strictly increasing in g and leaves every segment at least ceil(rows / 128)
// numbers, so tile s belongs to the last g whose number is not above s (a warp compares 32 segments at a time); at most G of
// the N / 128 + G numbers are empty.  A tile's 128 rows may reach into the next segment: the products of those rows are
// computed and not stored.
// SG_DW: the rows are cut into equal parts, whatever the segments; a CTA takes one block [128 features x bn columns] of the
// result over one part and finishes it for each segment that it meets there.  A segment that lies in one part is written at
// once; one that is cut leaves an fp32 partial per part (two per part at most: the segment cut at its start, the one cut at
// its end), added in ascending order by a second kernel: the order depends on the sizes alone.
//
// One persistent CTA per SM:
//   warp 0     loader: slices of 128 bytes along the contraction (64 rows for SG_DW) of both operands by bulk tensor copies into
//              a ring of shared-memory slots, 128-byte swizzle
//   warp 1     issues the tcgen05.mma of a slice into one of two accumulators in tensor memory.  SG_DW: the rows of a segment's
//              last slice that belong to the next one are overwritten with zeros first, in both operands (a zero in one would
//              not do: they may hold infinities)
//   warps 2-9  epilogue: accumulator -> registers -> swizzled staging -> whole rows to global memory, rows and columns that do
//              not exist left out
// fp32 (segment_gemm_f32_kernel): the same pieces of work, every value as three bf16 terms.
//
// Every wait has an iteration limit, as in linear_tma.cu.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "tc_common.cuh"

namespace gnn {

enum { SG_Y = 0, SG_DX = 1, SG_DW = 2, SG_I8 = 3 };

constexpr int SG_EPI_WARPS = 8;
constexpr int SG_THREADS = 32 * (2 + SG_EPI_WARPS);
constexpr int SG_MAX_STAGES = 8;
constexpr size_t SG_SMEM_MAX = 224 * 1024;      // dynamic; with the static part on its 1024-byte boundary: the 227 KB of a block
constexpr uint32_t SG_A_BYTES = 128 * 128;      // 128 rows of 128 bytes (SG_DW: two boxes of 64 features x 64 rows)
constexpr uint32_t SG_STAGING = 32 * 128;       // per epilogue warp
constexpr uint32_t SG_SW128 = 2;

struct SegGemmParams {
    const int64_t* seg_ptr;  // [G+1], or nullptr: one segment of all rows
    int G;
    int64_t N;
    int64_t units;           // tiles (SG_DW: parts x blocks of the result)
    int slices, contraction; // (not SG_DW) slices of the contraction, its elements
    int tiles_n, tiles_m;    // blocks of output columns; of features (SG_DW)
    int bn;                  // output columns of a tile: a multiple of 64, at most 256, fp32 128
    int stages, tmem_cols;
    int a_rows;              // rows of a box of A (not SG_DW): 128, fewer where there are fewer in all
    int64_t part_rows;       // SG_DW: rows of a part
    int rows_out, cols_out;  // output rows that exist (SG_DW: features), output columns
    void* out;               // rows cols_out elements apart; SG_DW: [G, rows_out, cols_out]
    int vec;                 // rows of out start on 16 bytes
    float* part;             // SG_DW: partials [2 * parts][rows_out][cols_out]
    const float* bias;       // [G, cols_out] or nullptr
    const float* sx;         // SG_I8: scales of the rows, of the columns
    const float* sw;
    int relu;
    int* status;
    int reset;
};

// rows [lo, hi) of segment g, kept inside [0, N) whatever seg_ptr holds
struct SegRows { int64_t lo, hi; int g; };
__device__ __forceinline__ int64_t seg_at(const SegGemmParams& P, int g) {
    if (!P.seg_ptr) return g > 0 ? P.N : 0;
    const int64_t v = P.seg_ptr[g];
    return v < 0 ? 0 : v > P.N ? P.N : v;
}
// last g in [0, G) with before(g) true for it (before is true up to some g); -1: none.  All lanes of a warp.
template <class F>
__device__ __forceinline__ int last_segment(int G, F before) {
    int lo = 0, hi = G;
    const int lane = threadIdx.x & 31;
    while (true) {
        const int step = (hi - lo + 31) >> 5;
        const int p = lo + lane * step;
        const int n = __popc(__ballot_sync(0xFFFFFFFFu, p < hi && before(p)));
        if (n == 0) return lo - 1;
        lo += (n - 1) * step;
        if (step == 1) return lo;
        hi = min(hi, lo + step);
    }
}
// tile number s -> its rows (hi <= lo: none)
__device__ __forceinline__ SegRows seg_tile(const SegGemmParams& P, int64_t s) {
    const int g = last_segment(P.G, [&](int q) { return seg_at(P, q) / TC_ROWS + q <= s; });
    if (g < 0) return {0, 0, 0};
    const int64_t a = seg_at(P, g), b = seg_at(P, g + 1);
    const int64_t lo = a + (s - (a / TC_ROWS + g)) * TC_ROWS;
    return {lo, lo + TC_ROWS < b ? lo + TC_ROWS : b, g};
}

__device__ __forceinline__ void sg_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
        : "memory");
}
// 8-bit integers: D = s32, A = B = s8, both K-major, 32 contraction elements
__host__ __device__ constexpr uint32_t make_idesc_i8(int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(TC_ROWS >> 4) << 24);
}
__device__ __forceinline__ void mma_i8_ss(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, {%5, %6, %7, %8}, p;\n\t"
        "}\n"
        :
        : "r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(0u), "r"(0u), "r"(0u), "r"(0u)
        : "memory");
}
__device__ __forceinline__ uint64_t policy_normal() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
    return p;
}
// Every role of a CTA walks the same pieces of work: body(rows of one segment, block of features, block of columns, part) until
// it says stop.
template <int MODE, class Body>
__device__ __forceinline__ void sg_walk(const SegGemmParams& P, Body body) {
    for (int64_t u = blockIdx.x; u < P.units; u += gridDim.x) {
        const int n = (int)(u % P.tiles_n);
        if constexpr (MODE != SG_DW) {
            const SegRows t = seg_tile(P, u / P.tiles_n);
            if (t.hi > t.lo && !body(t, 0, n, (int64_t)0)) return;
        } else {
            const int64_t v = u / P.tiles_n, part = v / P.tiles_m;
            const int64_t r0 = part * P.part_rows, r1 = r0 + P.part_rows < P.N ? r0 + P.part_rows : P.N;
            int g = last_segment(P.G, [&](int q) { return seg_at(P, q) <= r0; });
            for (g = g < 0 ? 0 : g; g < P.G; ++g) {
                const int64_t a = seg_at(P, g), b = seg_at(P, g + 1);
                if (a >= r1) break;
                const SegRows t = {a > r0 ? a : r0, b < r1 ? b : r1, g};
                if (t.hi > t.lo && !body(t, (int)(v % P.tiles_m), n, part)) return;
            }
        }
    }
}

__device__ __forceinline__ void sg_store(float* p, uint32_t bits) { *reinterpret_cast<uint32_t*>(p) = bits; }
__device__ __forceinline__ void sg_store(__nv_bfloat16* p, uint32_t bits) { *reinterpret_cast<uint16_t*>(p) = (uint16_t)bits; }

// One warp's 32 rows x 128 bytes from staging to global memory: columns [c0, c0 + 128 bytes), of which those under `cols` exist,
// rows under `rows`.  On 16-byte rows eight lanes send a row of 128 bytes; otherwise a lane sends an element, a row at a time.
template <typename T>
__device__ __forceinline__ void sg_rows_out(uint32_t stg, T* out, int64_t ld, int rows, int c0, int cols, bool vec, int lane) {
    constexpr int PER = 16 / sizeof(T), WIDE = 128 / sizeof(T);
    if (vec) {
        const int c = c0 + (lane & 7) * PER;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + (lane >> 3);
            if (r < rows && c < cols) {  // rows of out are whole chunks: so are cols
                uint4 v;
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                             : "r"(stg + (uint32_t)r * 128u + (uint32_t)(((lane & 7) ^ (r & 7)) << 4)) : "memory");
                *reinterpret_cast<uint4*>(out + r * ld + c) = v;
            }
        }
        return;
    }
    for (int r = 0; r < rows; ++r)
#pragma unroll
        for (int h = 0; h < WIDE / 32; ++h) {
            const int e = lane + 32 * h;
            if (c0 + e < cols) {
                const uint32_t at = stg + (uint32_t)r * 128u + (uint32_t)(((e / PER) ^ (r & 7)) << 4) + (uint32_t)(e % PER) * (uint32_t)sizeof(T);
                uint32_t v;
                if (sizeof(T) == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
                else { uint16_t h16; asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h16) : "r"(at) : "memory"); v = h16; }
                sg_store(out + r * ld + c0 + e, v);
            }
        }
}

// rows of no segment: zeros, by the epilogue warps (threads 64 .. 319 of each block)
template <typename T>
__device__ __forceinline__ void sg_zero_outside(const SegGemmParams& P, T* out) {
    const int64_t p0 = seg_at(P, 0) * P.cols_out, p1 = seg_at(P, P.G) * P.cols_out, end = P.N * P.cols_out;
    const int64_t me = (int64_t)blockIdx.x * (32 * SG_EPI_WARPS) + ((int)threadIdx.x - 64), all = (int64_t)gridDim.x * (32 * SG_EPI_WARPS);
    for (int64_t i = me; i < p0; i += all) out[i] = T(0.f);
    for (int64_t i = p1 + me; i < end; i += all) out[i] = T(0.f);
}

// 32 accumulator columns of this warp's 32 rows
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
    tmem_ld16(taddr, r);
    tmem_ld16(taddr + 16, r + 16);
}

template <int MODE, typename T>
__global__ void __launch_bounds__(SG_THREADS, 1)
segment_gemm_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const SegGemmParams P) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];  // swizzle atoms lie on 1024 bytes
    __shared__ __align__(8) uint64_t bars[2 * SG_MAX_STAGES + 4];  // full[S], empty[S], acc_full[2], acc_empty[2]
    __shared__ __align__(16) float s_cols[MODE == SG_I8 ? 2 : 1][256];                 // bias and column scales of the tile, zeros past the last
    __shared__ uint32_t tmem_base_slot;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int S = P.stages, bn = P.bn;
    const uint32_t base = smem_u32(smem_raw);
    if (base & 1023u) {  // (never: the array's own alignment)
        if (tid == 0) atomicExch(P.status, 7);
        return;
    }
    const uint32_t b_bytes = (uint32_t)bn * 128u;
    const uint32_t slot_bytes = SG_A_BYTES + b_bytes;
    const uint32_t stage0 = base, ring0 = base + SG_EPI_WARPS * SG_STAGING;
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty = [&](int s) { return bar0 + 8u * (uint32_t)(SG_MAX_STAGES + s); };
    auto acc_full = [&](uint32_t a) { return bar0 + 8u * (uint32_t)(2 * SG_MAX_STAGES + a); };
    auto acc_empty = [&](uint32_t a) { return bar0 + 8u * (uint32_t)(2 * SG_MAX_STAGES + 2 + a); };

    if (tid == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (uint32_t a = 0; a < 2; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), SG_EPI_WARPS); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapA)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapB)) : "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(&tmem_base_slot), (uint32_t)P.tmem_cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait_exclusive();
    if (P.reset && blockIdx.x == 0 && tid == 0) *P.status = 0;
    const uint32_t tmem_base = tmem_base_slot;
    const uint32_t acc_cols = (uint32_t)bn;
    bool failed = false;

    auto walk = [&](auto body) { sg_walk<MODE>(P, body); };
    auto slices_of = [&](const SegRows& t) { return MODE == SG_DW ? (int)((t.hi - t.lo + 63) >> 6) : P.slices; };

    if (warp == 0) {
        const uint64_t keep = policy_evict_last(), once = P.tiles_n > 1 || P.tiles_m > 1 ? policy_normal() : policy_evict_first();
        uint32_t it = 0;
        const uint32_t a_box = MODE == SG_DW ? SG_A_BYTES : (uint32_t)P.a_rows * 128u;
        walk([&](const SegRows& t, int mb, int nb, int64_t) {
            const int slices = slices_of(t);
            for (int j = 0; j < slices; ++j, ++it) {
                const int s = (int)(it % (uint32_t)S);
                bool ok = true;
                if (lane == 0) {
                    ok = mbar_wait_bounded(empty(s), ((it / (uint32_t)S) & 1u) ^ 1u);
                    if (ok) {
                        mbar_arrive_expect_tx(full(s), a_box + b_bytes);
                        const uint32_t a0 = ring0 + (uint32_t)s * slot_bytes, b0 = a0 + SG_A_BYTES;
                        if constexpr (MODE == SG_DW) {
                            const int row = (int)(t.lo + (int64_t)j * 64);
                            for (int h = 0; h < 2; ++h) sg_load(a0 + (uint32_t)h * 8192u, &mapA, mb * 128 + h * 64, row, 0, full(s), once);
                            for (int h = 0; h < bn / 64; ++h) sg_load(b0 + (uint32_t)h * 8192u, &mapB, nb * bn + h * 64, row, 0, full(s), once);
                        } else {
                            constexpr int STEP = MODE == SG_I8 ? 128 : 64;  // elements of 128 bytes
                            sg_load(a0, &mapA, j * STEP, (int)t.lo, 0, full(s), once);
                            if constexpr (MODE == SG_Y)
                                for (int h = 0; h < bn / 64; ++h) sg_load(b0 + (uint32_t)h * 8192u, &mapB, nb * bn + h * 64, j * 64, t.g, full(s), keep);
                            else
                                sg_load(b0, &mapB, j * STEP, nb * bn, t.g, full(s), keep);
                        }
                    }
                }
                if (!__shfl_sync(0xFFFFFFFFu, (int)ok, 0)) { failed = true; return false; }
            }
            return true;
        });
        if (failed && lane == 0) {
            // do not leave while copies into this CTA's shared memory may still be in flight
            const uint32_t first = it > (uint32_t)S ? it - (uint32_t)S : 0u;
            for (uint32_t i = first; i < it; ++i) mbar_wait_bounded(full((int)(i % (uint32_t)S)), (i / (uint32_t)S) & 1u);
        }
    } else if (warp == 1) {
        const uint32_t idesc = MODE == SG_I8 ? make_idesc_i8(bn) : make_idesc(bn, MODE != SG_DX, MODE == SG_DW);
        uint32_t it = 0, lt = 0;
        walk([&](const SegRows& t, int, int, int64_t) {
            const uint32_t a = lt & 1u;
            const uint32_t dacc = tmem_base + a * acc_cols;
            const int slices = slices_of(t);
            bool ok = lane != 0 || mbar_wait_bounded(acc_empty(a), ((lt >> 1) & 1u) ^ 1u);
            for (int j = 0; j < slices; ++j, ++it) {
                const int s = (int)(it % (uint32_t)S);
                const uint32_t a0 = ring0 + (uint32_t)s * slot_bytes, b0 = a0 + SG_A_BYTES;
                if (lane == 0 && ok) ok = mbar_wait_bounded(full(s), (it / (uint32_t)S) & 1u);
                if (!__shfl_sync(0xFFFFFFFFu, (int)ok, 0)) { failed = true; return false; }
                if constexpr (MODE == SG_DW) {
                    const int have = (int)(t.hi - t.lo - (int64_t)j * 64);
                    if (have < 64) {  // rows of the next segment: 128 bytes each, from `have` to the end of every box
                        mbar_wait_bounded(full(s), (it / (uint32_t)S) & 1u);  // (has completed: orders every lane's stores behind the copies)
                        for (int box = 0; box < 2 + bn / 64; ++box)
                            for (uint32_t o = (uint32_t)have * 128u + (uint32_t)lane * 16u; o < 8192u; o += 512u)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a0 + (uint32_t)box * 8192u + o), "r"(0u) : "memory");
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                }
                if (lane == 0) {
                    tc_fence_after();
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) {
                        // K-major: rows 128 bytes apart, groups of 8 rows 1024, a k-step 32 bytes along the row.  MN-major: 16
                        // contraction rows of 128 bytes a k-step, boxes of 64 columns 8192 bytes apart
                        const uint64_t ad = MODE == SG_DW ? make_smem_desc(a0 + (uint32_t)kk * 2048u, 8192, 1024, SG_SW128)
                                                          : make_smem_desc(a0 + (uint32_t)kk * 32u, 16, 1024, SG_SW128);
                        const uint64_t bd = MODE == SG_DW || MODE == SG_Y ? make_smem_desc(b0 + (uint32_t)kk * 2048u, 8192, 1024, SG_SW128)
                                                                          : make_smem_desc(b0 + (uint32_t)kk * 32u, 16, 1024, SG_SW128);
                        const uint32_t more = j > 0 || kk > 0;
                        if constexpr (MODE == SG_I8) mma_i8_ss(dacc, ad, bd, idesc, more);
                        else mma_bf16_ss(dacc, ad, bd, idesc, more);
                    }
                    mma_commit(empty(s));
                }
                __syncwarp();
            }
            if (lane == 0) mma_commit(acc_full(a));
            ++lt;
            return true;
        });
    } else {
        const int ew = warp - 2, quarter = warp & 3, half = ew >> 2;  // tensor-memory lanes 32 * (warp % 4)..: hardware rule
        const uint32_t stg = stage0 + (uint32_t)ew * SG_STAGING;
        uint32_t lt = 0;
        int staged_g = -1, staged_n = -1;
        walk([&](const SegRows& t, int mb, int nb, int64_t part) {
            const uint32_t a = lt & 1u;
            if (MODE != SG_DW && (P.bias || MODE == SG_I8) && (t.g != staged_g || nb != staged_n)) {  // the same in all epilogue warps
                const int c = tid - 64, col = nb * bn + c;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                s_cols[0][c] = P.bias && c < bn && col < P.cols_out ? P.bias[(int64_t)t.g * P.cols_out + col] : 0.f;
                if constexpr (MODE == SG_I8) s_cols[1][c] = c < bn && col < P.cols_out ? P.sw[col] : 0.f;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                staged_g = t.g;
                staged_n = nb;
            }
            if (!mbar_wait_bounded(acc_full(a), (lt >> 1) & 1u)) { failed = true; return false; }
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + a * acc_cols;
            const int64_t left = MODE == SG_DW ? (int64_t)P.rows_out - mb * 128 - quarter * 32 : t.hi - t.lo - quarter * 32;
            const int rows = (int)(left < 32 ? left : 32);
            const bool cut = MODE == SG_DW && (seg_at(P, t.g) != t.lo || seg_at(P, t.g + 1) != t.hi);
            const int c_base = nb * bn, c_end = P.cols_out;
            float sx = 0.f;
            if (MODE == SG_I8 && lane < rows) sx = P.sx[t.lo + quarter * 32 + lane];
            // 32 columns at c -> fp32 values
            auto fetch = [&](int c, float* f) {
                uint32_t r[32];
                tmem_ld32(taddr + (uint32_t)c, r);
                tmem_ld_wait();
#pragma unroll
                for (int q = 0; q < 32; ++q) f[q] = MODE == SG_I8 ? (float)(int)r[q] : __uint_as_float(r[q]);
                if constexpr (MODE == SG_I8) {
#pragma unroll
                    for (int q = 0; q < 32; q += 4) {
                        const float4 w = *reinterpret_cast<const float4*>(&s_cols[1][c + q]);
                        f[q] *= sx * w.x; f[q + 1] *= sx * w.y; f[q + 2] *= sx * w.z; f[q + 3] *= sx * w.w;
                    }
                }
                if (MODE != SG_DW && P.bias) {
#pragma unroll
                    for (int q = 0; q < 32; q += 4) {
                        const float4 b = *reinterpret_cast<const float4*>(&s_cols[0][c + q]);
                        f[q] += b.x; f[q + 1] += b.y; f[q + 2] += b.z; f[q + 3] += b.w;
                    }
                }
                if (MODE != SG_DW && P.relu) {
#pragma unroll
                    for (int q = 0; q < 32; ++q) f[q] = f[q] < 0.f ? 0.f : f[q];  // NaN stays
                }
            };
            auto send = [&](auto* out, int64_t ld, bool vec) {
                using O = typename std::remove_pointer<decltype(out)>::type;
                constexpr int WIDE = 128 / sizeof(O), CH = 32 * sizeof(O) / 16;  // columns of a staging row; chunks of 32 columns
                for (int cb = half; cb * WIDE < bn; cb += 2) {
                    if (c_base + cb * WIDE >= c_end || rows <= 0) break;  // the whole warp
                    __syncwarp();
#pragma unroll
                    for (int h = 0; h < WIDE / 32; ++h) {
                        float f[32];
                        fetch(cb * WIDE + h * 32, f);
#pragma unroll
                        for (int q = 0; q < CH; ++q) {
                            const uint4 v = Chunk<O>::pack(f + q * Chunk<O>::N);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stg + (uint32_t)lane * 128u + (uint32_t)(((h * CH + q) ^ (lane & 7)) << 4)),
                                         "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
                        }
                    }
                    __syncwarp();
                    sg_rows_out<O>(stg, out, ld, rows, c_base + cb * WIDE, c_end, vec, lane);
                }
            };
            if constexpr (MODE == SG_DW) {
                const int64_t off = (int64_t)(mb * 128 + quarter * 32) * P.cols_out;
                const int64_t size = (int64_t)P.rows_out * P.cols_out;
                if (cut) {
                    // cut at the part's start: partial 2p, else (at its end) 2p + 1
                    const int64_t which = 2 * part + (seg_at(P, t.g) >= part * P.part_rows ? 1 : 0);
                    send(P.part + which * size + off, P.cols_out, P.cols_out % 4 == 0);
                } else {
                    send((T*)P.out + t.g * size + off, P.cols_out, P.vec != 0);
                }
            } else {
                send((T*)P.out + (t.lo + quarter * 32) * P.cols_out, P.cols_out, P.vec != 0);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty(a));
            ++lt;
            return true;
        });
        if (MODE == SG_Y || MODE == SG_DX) sg_zero_outside(P, (T*)P.out);
    }
    if (failed) atomicExch(P.status, 7);  // GNN_ERR_TIMEOUT
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, (uint32_t)P.tmem_cols);
}

// [planes, rows, cols] of bf16 (or bytes), rows ld elements apart, planes directly after one another; box = 128 bytes x box_rows
// rows of one plane, swizzled; out-of-range reads give zeros (linear_tma.cu)
// type: 0 bf16, 1 bytes, 2 fp32
bool make_map_planes(CUtensorMap* m, const void* ptr, int type, int64_t planes, int64_t rows, int64_t cols, int64_t ld, int box_rows);
bool tensor_map_encoder_available();
// SG_Y, SG_DX or SG_DW of fp32 (segment_gemm_f32.cu); slot: of allow_big_smem
gnn_status segment_gemm_f32(const char* who, int mode, int slot, const CUtensorMap& mapA, const CUtensorMap& mapB, SegGemmParams& P, cudaStream_t st);

// output columns of a tile: as few blocks of at most `most` as cover them, evened out, in steps of 64; halved while there are
// fewer tiles than SMs (a tile's weights then arrive through more SMs)
inline int sg_block(int cols, int most, int64_t row_tiles) {
    const int blocks = (cols + most - 1) / most;
    int bn = ((cols + blocks - 1) / blocks + 63) / 64 * 64;
    while (bn > 64 && row_tiles * ((cols + bn - 1) / bn) < 148) bn = (bn / 2 + 63) / 64 * 64;
    return bn;
}

template <int MODE, typename T>
static gnn_status sg_launch(const char* who, int which, const CUtensorMap& mapA, const CUtensorMap& mapB, SegGemmParams& P, cudaStream_t st) {
    const auto kernel = segment_gemm_kernel<MODE, T>;
    const gnn_status rc = allow_big_smem(who, (const void*)kernel, which, SG_SMEM_MAX);
    if (rc != GNN_OK) return rc;
    const size_t fixed = SG_EPI_WARPS * SG_STAGING, slot = SG_A_BYTES + (size_t)P.bn * 128;
    int stages = (int)((SG_SMEM_MAX - fixed) / slot);
    P.stages = stages > SG_MAX_STAGES ? SG_MAX_STAGES : stages;
    int cols = 32;
    while (cols < 2 * P.bn) cols <<= 1;
    P.tmem_cols = cols;
    launch_overlapped(kernel, dim3((unsigned)(P.units < 148 ? P.units : 148)), dim3(SG_THREADS), fixed + (size_t)P.stages * slot, st, mapA, mapB, P);
    GNN_CHECK_LAUNCH(who);
    return GNN_OK;
}

}  // namespace gnn
