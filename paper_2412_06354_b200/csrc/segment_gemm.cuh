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
// Tiles of SG_Y, SG_DX and SG_I8: 128 rows of ONE segment x bn output columns.  A block number leads to its segment without a
// prefix sum: floor(seg_ptr[g] / R) + g is strictly increasing in g and leaves every segment at least ceil(rows / R) numbers, so
// block s of R rows belongs to the last g whose number is not above s (a warp compares 32 segments at a time); at most G of
// the N / R + G numbers are empty.  A tile's 128 rows may reach into the next segment: the products of those rows are
// computed and not stored.
//   ranges > 0: every CTA takes one block of columns of a range of consecutive blocks of 32 rows, equally many for each, and cuts
//               it into tiles as the segments ask.  Its weights stay in shared memory as long as the segment does (where the
//               contraction is short enough: `resident` buffers of them), so that the ring brings rows alone, and CTAs end together:
//               170,000 x 128 -> 128, 1334 tiles dealt out to 148 SMs one by one: a tenth round for a few.
//   otherwise:  tiles of 128 rows dealt out, all columns of a tile side by side: neighbouring CTAs share a segment's weights in L2, which
//               could not hold all segments' at once; and where there are few rows.
//   pair:       such a tile is 256 rows, a slice of weights serves both halves, one accumulator each.  An SM takes about 60 bytes a
//               cycle from L2: 48 KB a slice of 128 x 256 are 820 cycles of copies beside 512 of products, 64 KB of 256 x 256 are 1090
//               beside 1024.  The epilogue no longer runs beside the next tile's products, which long contractions make up for.
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
//   warps 2-17 epilogue: accumulator -> registers -> swizzled staging -> rows of 64 bytes to global memory, rows and columns that
//              do not exist left out.  (Eight warps with 128 bytes: 8-bit product of 170,000 x 256 -> 256 40 us, of which 20 without
//              any epilogue; sixteen 32 us, and 29 with the bulk stores below.)
// Measured in short runs (in runs of seconds, under the power cap): 170,000 x 128 -> 128 over 12 segments 18.5 us (20.5; 4.7 TB/s: HBM, and 4 us of start
// and end), 65,536 x 1024 -> 1024 over 64 134 us (157; 1.02 and 0.88 PFLOP/s: copies from L2), gradients of 100,000 x 256 x 256 over 12 58 us (62),
// 8 bits 170,000 x 256 -> 256 to bf16 29 us (4.5 TB/s), 16,384 x 2048 -> 2048 to fp32 65.5 us (2.1e15 operations a second; with the rounding of its
// rows 96, 109 in long runs).
// fp32 (segment_gemm_f32_kernel): the same pieces of work, every value as three bf16 terms.
//
// Every wait has an iteration limit, as in linear_tma.cu.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "tc_common.cuh"

namespace gnn {

enum { SG_Y = 0, SG_DX = 1, SG_DW = 2, SG_I8 = 3 };

constexpr int SG_EPI_WARPS = 16;
constexpr int SG_THREADS = 32 * (2 + SG_EPI_WARPS);
constexpr int SG_MAX_STAGES = 10;
constexpr size_t SG_SMEM_MAX = 224 * 1024;      // dynamic; with the static part on its 1024-byte boundary: the 227 KB of a block
constexpr uint32_t SG_A_BYTES = 128 * 128;      // 128 rows of 128 bytes (SG_DW: two boxes of 64 features x 64 rows)
constexpr uint32_t SG_STAGING = 32 * 64;        // per epilogue warp: 32 rows of 64 bytes
constexpr uint32_t SG_SW128 = 2;

struct SegGemmParams {
    const int64_t* seg_ptr;  // [G+1], or nullptr: one segment of all rows
    int G;
    int64_t N;
    int64_t units;           // tiles, or ranges x blocks of columns (SG_DW: parts x blocks of the result)
    int ranges, resident;    // see above
    int pair;                // tiles of 256 rows: both accumulators at once
    unsigned per_range, longer;
    int slices, contraction; // (not SG_DW) slices of the contraction, its elements
    int tiles_n, tiles_m;    // blocks of output columns; of features (SG_DW)
    int bn;                  // output columns of a tile: a multiple of 64, at most 256, fp32 128
    int stages, tmem_cols;
    int a_rows;              // rows of a box of A (not SG_DW): 128, fewer where there are fewer in all
    int64_t part_rows;       // SG_DW: rows of a part
    int rows_out, cols_out;  // output rows that exist (SG_DW: features), output columns
    void* out;               // rows cols_out elements apart; SG_DW: [G, rows_out, cols_out]
    int vec;                 // rows of out start on 16 bytes
    int bulk;                // whole boxes of 32 rows x 64 bytes leave by bulk stores through mapO (SG_DW: of the partials)
    float* part;             // SG_DW: partials [2 * parts][rows_out][cols_out]
    const float* bias;       // [G, cols_out] or nullptr
    const float* sx;         // SG_I8: scales of the rows, of the columns
    const float* sw;
    int relu;
    int* status;
    int reset;
};

// rows [lo, hi) of segment g, kept inside [0, N) and behind a whatever seg_ptr holds
struct SegRows { int64_t lo, hi; int g; int64_t a, b; };  // a, b: all rows of the segment
__device__ __forceinline__ int64_t seg_at(const SegGemmParams& P, int g) {
    if (!P.seg_ptr) return g > 0 ? P.N : 0;
    const int64_t v = P.seg_ptr[g];
    return v < 0 ? 0 : v > P.N ? P.N : v;
}
// Last g in [0, G) with before(g, seg_ptr[g]) true for it (before is true up to some g), and its rows; g = -1: none.  All lanes of a
// warp; the last step has the bounds at hand, so that up to 31 segments take one round of loads.
struct SegFound { int g; int64_t a, b; };
template <class F>
__device__ __forceinline__ SegFound last_segment(const SegGemmParams& P, F before) {
    int lo = 0, hi = P.G;
    const int lane = threadIdx.x & 31;
    while (true) {
        const int step = (hi - lo + 31) >> 5;
        const int p = lo + lane * step;
        const int64_t v = p <= P.G ? seg_at(P, p) : P.N;
        const int n = __popc(__ballot_sync(0xFFFFFFFFu, p < hi && before(p, v)));
        if (n == 0) return {lo - 1, 0, 0};
        if (step == 1) {
            const int g = lo + n - 1;
            const int64_t a = __shfl_sync(0xFFFFFFFFu, v, n - 1), b = __shfl_sync(0xFFFFFFFFu, v, n & 31);
            return {g, a, n < 32 ? b : seg_at(P, g + 1)};
        }
        lo += (n - 1) * step;
        hi = min(hi, lo + step);
    }
}
// Block number s of 2^shift rows -> its segment and first row, for ascending s: the segment of the last one is kept, so that most
// are two comparisons and an addition.  (Searching anew for each, with 64-bit divisions, took the loader 1000 cycles a tile.)
struct SegCursor {
    int g;
    int64_t a, b, first, next;  // rows of segment g, its block numbers
    __device__ __forceinline__ SegCursor() : g(-1), a(0), b(0), first(0), next(0) {}
    // first row of block s; g < 0: before the first segment
    __device__ __forceinline__ int64_t at(const SegGemmParams& P, int64_t s, int shift) {
        if (s >= next) {
            const SegFound f = last_segment(P, [&](int q, int64_t v) { return (v >> shift) + q <= s; });
            if (f.g < 0) return 0;
            g = f.g;
            a = f.a;
            b = f.b;
            first = (a >> shift) + g;
            next = (b >> shift) + g + 1;  // (of the next segment; not above the true bound where seg_ptr descends)
        }
        return a + ((s - first) << shift);
    }
};

// a bounded wait of a whole warp, with one answer
__device__ __forceinline__ bool sg_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, parity)); }
// a meeting of as many warps as bar counts, the met-th at this barrier: as bar.sync, but with a limit (a warp that gave up does not come)
__device__ __forceinline__ bool sg_meet(uint32_t bar, uint32_t met) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
    return sg_wait(bar, met & 1u);
}
// a place in a ring of n slots and the parity of its round (counted, not divided: n is known at run time only)
struct SgRing {
    uint32_t n, s, parity, uses;
    __device__ __forceinline__ explicit SgRing(int slots) : n((uint32_t)slots), s(0), parity(0), uses(0) {}
    __device__ __forceinline__ void next() {
        ++uses;
        if (++s == n) { s = 0; parity ^= 1u; }
    }
    // waits for the last use of every slot: bar(slot)
    template <class F>
    __device__ __forceinline__ void drain(F bar) const {
        for (uint32_t q = 0; q < n; ++q)
            if (q < s || uses >= n) mbar_wait_bounded(bar(q), q < s ? parity : parity ^ 1u);
    }
};
// What one thread of a warp does, called by the whole warp: the election stands in the instruction itself, so that the control flow
// around it stays that of a whole warp.  (As a branch of lane 0 around loops of them, copies took 250 cycles each to issue and MMAs
// 85.)  The same thread is elected every time.
#define SG_ELECT "{\n\t.reg .pred p, q;\n\telect.sync _|p, 0xFFFFFFFF;\n\t"
__device__ __forceinline__ void sg_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar, uint64_t policy) {
    asm volatile(SG_ELECT
                 "@p cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;\n\t}"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void sg_expect(uint32_t bar, uint32_t bytes) {
    asm volatile(SG_ELECT "@p mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void sg_commit(uint32_t bar) {
    asm volatile(SG_ELECT "@p tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
// D (+)= A B: A in shared memory (a descriptor) or in tensor memory (an address)
__device__ __forceinline__ void sg_mma_bf16(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(SG_ELECT "setp.ne.b32 q, %4, 0;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, q;\n\t}"
                 ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void sg_mma_bf16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(SG_ELECT "setp.ne.b32 q, %4, 0;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, q;\n\t}"
                 ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void sg_mma_i8(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(SG_ELECT "setp.ne.b32 q, %4, 0;\n\t@p tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, q;\n\t}"
                 ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// 8-bit integers: D = s32, A = B = s8, both K-major, 32 contraction elements
__host__ __device__ constexpr uint32_t make_idesc_i8(int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(TC_ROWS >> 4) << 24);
}
__device__ __forceinline__ uint64_t policy_normal() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
    return p;
}
// seg_ptr on its way to L2 while the kernel before still runs (a hint: nothing of it is used before pdl_wait)
__device__ __forceinline__ void sg_touch(const SegGemmParams& P) {
    if (P.seg_ptr && blockIdx.x == 0 && (int)threadIdx.x * 16 <= P.G) asm volatile("prefetch.global.L2 [%0];" ::"l"(P.seg_ptr + threadIdx.x * 16));
}

// Every role of a CTA walks the same pieces of work: body(rows of one segment, block of features, block of columns, part) until
// it says stop.
template <int MODE, class Body>
__device__ __forceinline__ void sg_walk(const SegGemmParams& P, Body body) {
    if (MODE != SG_DW && P.ranges > 0) {
        // unit = range of consecutive blocks of 32 rows * tiles_n + block of columns; a range is per_range blocks, the first ones of a
        // remainder one more.  (No 64-bit division: a microsecond of a CTA's start.)
        for (unsigned u = blockIdx.x; u < (unsigned)P.units; u += gridDim.x) {
            const unsigned r = P.tiles_n == 1 ? u : u / (unsigned)P.tiles_n;
            const int n = (int)(u - r * (unsigned)P.tiles_n);
            const int64_t s0 = r * P.per_range + (r < P.longer ? r : P.longer), s1 = s0 + P.per_range + (r < P.longer ? 1u : 0u);
            SegCursor at;
            for (int64_t s = s0; s < s1;) {
                const int64_t lo = at.at(P, s, 5);
                if (at.g < 0 || lo < at.a || lo >= at.b) {  // rows of no segment before the first one, the empty block at a segment's end (lo < a: seg_ptr descends)
                    s = at.g < 0 ? (seg_at(P, 0) >> 5) > s ? (seg_at(P, 0) >> 5) : s + 1 : at.next > s ? at.next : s + 1;
                    continue;
                }
                int64_t hi = lo + TC_ROWS < at.b ? lo + TC_ROWS : at.b;
                const int64_t end = at.a + ((s1 - at.first) << 5);  // what follows belongs to the next range
                if (hi > end) hi = end;
                if (!body(SegRows{lo, hi, at.g, at.a, at.b}, 0, n, (int64_t)0)) return;
                s = s + (TC_ROWS >> 5) < at.next ? s + (TC_ROWS >> 5) : at.next > s ? at.next : s + 1;
            }
        }
    } else if constexpr (MODE != SG_DW) {
        // unit = number of a tile of 128 (pair: 256) rows * tiles_n + block of columns
        const unsigned nn = (unsigned)P.tiles_n, ds = gridDim.x / nn, dn = gridDim.x % nn;
        unsigned n = blockIdx.x % nn;
        int64_t s = blockIdx.x / nn;
        const int shift = P.pair ? 8 : 7;
        SegCursor at;
        for (int64_t u = blockIdx.x; u < P.units; u += gridDim.x) {
            const int64_t lo = at.at(P, s, shift), hi = lo + ((int64_t)1 << shift);
            const SegRows t = {lo, hi < at.b ? hi : at.b, at.g, at.a, at.b};
            if (at.g >= 0 && t.lo >= at.a && t.hi > t.lo && !body(t, 0, (int)n, (int64_t)0)) return;  // (lo < a: seg_ptr descends)
            s += ds;
            n += dn;
            if (n >= nn) { n -= nn; ++s; }
        }
    } else {
        const unsigned tn = (unsigned)P.tiles_n, tm = (unsigned)P.tiles_m;
        for (unsigned u = blockIdx.x; u < (unsigned)P.units; u += gridDim.x) {  // (parts x blocks of the result: far below 2^31)
            const unsigned v = u / tn, w = v / tm;
            const int n = (int)(u - v * tn), mb = (int)(v - w * tm);
            const int64_t part = w;
            const int64_t r0 = part * P.part_rows, r1 = r0 + P.part_rows < P.N ? r0 + P.part_rows : P.N;
            SegFound f = last_segment(P, [&](int, int64_t v) { return v <= r0; });
            int g = f.g;
            int64_t a = f.a, b = f.b;
            if (g < 0) { g = 0; a = seg_at(P, 0); b = seg_at(P, 1); }
            for (; g < P.G; ++g, a = b, b = g < P.G ? seg_at(P, g + 1) : b) {
                if (a >= r1) break;
                const SegRows t = {a > r0 ? a : r0, b < r1 ? b : r1, g, a, b};
                if (t.hi > t.lo && !body(t, mb, n, part)) return;
            }
        }
    }
}

__device__ __forceinline__ void sg_store(float* p, uint32_t bits) { *reinterpret_cast<uint32_t*>(p) = bits; }
__device__ __forceinline__ void sg_store(__nv_bfloat16* p, uint32_t bits) { *reinterpret_cast<uint16_t*>(p) = (uint16_t)bits; }

// One warp's 32 rows x 64 bytes: row `lane` to staging as four chunks of 16 bytes, chunk c at c ^ (row / 2) % 4 (eight rows then fall on
// different banks), and from there to global memory: columns from c0, of which those under `cols` exist, rows under `rows`.  On
// 16-byte rows four lanes send a row's 64 bytes; otherwise a lane sends an element, a row (bf16) or two (fp32) at a time.
__device__ __forceinline__ uint32_t sg_staged(uint32_t stg, int r, int c) { return stg + (uint32_t)r * 64u + (uint32_t)((c ^ ((r >> 1) & 3)) << 4); }
__device__ __forceinline__ void sg_stage(uint32_t stg, int lane, int c, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(sg_staged(stg, lane, c)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
template <typename T>
__device__ __forceinline__ void sg_rows_out(uint32_t stg, T* out, int64_t ld, int rows, int c0, int cols, bool vec, int lane) {
    constexpr int PER = 16 / sizeof(T), WIDE = 64 / sizeof(T);
    if (vec) {
        const int c = c0 + (lane & 3) * PER, r0 = lane >> 2;
        T* to = out + r0 * ld + c;
        const int64_t step = 8 * ld;
        uint4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)  // (row + 8: the same place of its chunks)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w) : "r"(sg_staged(stg, r0, lane & 3) + (uint32_t)i * 512u) : "memory");
        if (rows == 32 && c0 + WIDE <= cols) {
#pragma unroll
            for (int i = 0; i < 4; ++i, to += step) *reinterpret_cast<uint4*>(to) = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i, to += step)
                if (r0 + 8 * i < rows && c < cols) *reinterpret_cast<uint4*>(to) = v[i];  // rows of out are whole chunks: so are cols
        }
        return;
    }
    const int e = lane % WIDE;
    if (c0 + e >= cols) return;
    for (int r = lane / WIDE; r < rows; r += 32 / WIDE) {
        const uint32_t at = sg_staged(stg, r, e / PER) + (uint32_t)(e % PER) * (uint32_t)sizeof(T);
        uint32_t v;
        if (sizeof(T) == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
        else { uint16_t h16; asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h16) : "r"(at) : "memory"); v = h16; }
        sg_store(out + r * ld + c0 + e, v);
    }
}

// ... or, where all 32 rows exist, by one bulk tensor store (columns past the last are clipped; the places of the chunks are those of
// the copy engine's 64-byte swizzle), which runs on while the warp does: sg_staging_free before the next use, sg_stores_done at the end.
// (65,536 x 1024 -> 1024 over 64 segments 138 -> 133 us, 170k x 256 -> 256 in 8 bits 32 -> 29 us.)
__device__ __forceinline__ void sg_box_out(uint32_t stg, const CUtensorMap* map, int x, int y, int lane) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(0), "r"(stg) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
__device__ __forceinline__ void sg_staging_free(int lane) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
}
__device__ __forceinline__ void sg_stores_done(int lane) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// rows of no segment: zeros, by the epilogue warps (threads from 64 on)
template <int WARPS, typename T>
__device__ __forceinline__ void sg_zero_outside(const SegGemmParams& P, T* out) {
    const int64_t p0 = seg_at(P, 0) * P.cols_out, p1 = seg_at(P, P.G) * P.cols_out, end = P.N * P.cols_out;
    const int64_t me = (int64_t)blockIdx.x * (32 * WARPS) + ((int)threadIdx.x - 64), all = (int64_t)gridDim.x * (32 * WARPS);
    for (int64_t i = me; i < p0; i += all) out[i] = T(0.f);
    for (int64_t i = p1 + me; i < end; i += all) out[i] = T(0.f);
}

// SG_I8: sum * sx * sw + b, roundings of the sum, of its product with sx, of the result.  A sum is under 2^31: from |sx| of 2^96 on (rows of
// 1e31 and more) that product may pass the largest number where the result does not; there 2^-32 of it meets 2^32 sw, in which a
// scale that has no room for that becomes the largest number (the result has none either, unless the sum is 0).  The same digits.
__device__ __forceinline__ bool sg_i8_wide(float sx) { return fabsf(sx) > 0x1p96f; }
__device__ __forceinline__ float sg_i8_value(int sum, float sx, float sw, float b) { return fmaf((float)sum * sx, sw, b); }
__device__ __forceinline__ float sg_i8_wide_value(int sum, float sx, float sw, float b) {
    const float w = fabsf(sw) > 0x1p95f && fabsf(sw) < INFINITY ? copysignf(3.402823466e38f, sw) : sw * 0x1p32f;
    return fmaf((float)sum * (sx * 0x1p-32f), w, b);
}

// a chunk of 16 bytes, not under floor: 0 (relu) or -inf, twice as bf16; a NaN stays.  (Of rounded values, as of the sums.)
__device__ __forceinline__ uint4 sg_pack(const float* f, const float*, uint32_t floor) {
    float g[4] = {f[0], f[1], f[2], f[3]};
#pragma unroll
    for (int q = 0; q < 4; ++q) asm("max.NaN.f32 %0, %0, %1;" : "+f"(g[q]) : "f"(__uint_as_float(floor & 0xFFFF0000u)));
    return Chunk<float>::pack(g);
}
__device__ __forceinline__ uint4 sg_pack(const float* f, const __nv_bfloat16*, uint32_t floor) {
    const uint4 v = Chunk<__nv_bfloat16>::pack(f);
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(w[q]) : "r"(floor));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int MODE, typename T>
__global__ void __launch_bounds__(SG_THREADS, 1)
segment_gemm_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ CUtensorMap mapO,
                    const SegGemmParams P) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];  // swizzle atoms lie on 1024 bytes
    __shared__ __align__(8) uint64_t bars[2 * SG_MAX_STAGES + 9];  // full[S], empty[S], acc_full[2], acc_empty[2], b_full[2], b_empty[2], meet
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
    const int nres = P.resident;  // (SG_DW: 0)
    const bool pair = MODE != SG_DW && P.pair != 0;
    const uint32_t a_bytes = pair ? 2 * SG_A_BYTES : SG_A_BYTES, slot_bytes = a_bytes + (nres ? 0u : b_bytes), b_tile = (uint32_t)P.slices * b_bytes;
    const uint32_t stage0 = base, res0 = base + SG_EPI_WARPS * SG_STAGING, ring0 = res0 + (uint32_t)nres * b_tile;
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty = [&](int s) { return bar0 + 8u * (uint32_t)(SG_MAX_STAGES + s); };
    auto acc_full = [&](uint32_t a) { return bar0 + 8u * (uint32_t)(2 * SG_MAX_STAGES + a); };
    auto acc_empty = [&](uint32_t a) { return bar0 + 8u * (uint32_t)(2 * SG_MAX_STAGES + 2 + a); };
    auto b_full = [&](uint32_t b) { return bar0 + 8u * (uint32_t)(2 * SG_MAX_STAGES + 4 + b); };
    auto b_empty = [&](uint32_t b) { return bar0 + 8u * (uint32_t)(2 * SG_MAX_STAGES + 6 + b); };
    const uint32_t meet = bar0 + 8u * (uint32_t)(2 * SG_MAX_STAGES + 8);

    if (tid == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (uint32_t a = 0; a < 2; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), SG_EPI_WARPS); mbar_init(b_full(a), 1); mbar_init(b_empty(a), 1); }
        mbar_init(meet, SG_EPI_WARPS);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapA)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapB)) : "memory");
    }
    sg_touch(P);
    if (warp == 1) tmem_alloc(smem_u32(&tmem_base_slot), (uint32_t)P.tmem_cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait_exclusive();  // (set up early, the next kernel's blocks cost these more than its start saves: dW 36 -> 39 us)
    if (P.reset && blockIdx.x == 0 && tid == 0) *P.status = 0;
    const uint32_t tmem_base = tmem_base_slot;
    const uint32_t acc_cols = (uint32_t)bn;
    bool failed = false;

    auto walk = [&](auto body) { sg_walk<MODE>(P, body); };
    auto slices_of = [&](const SegRows& t) { return MODE == SG_DW ? (int)((t.hi - t.lo + 63) >> 6) : P.slices; };

    if (warp == 0) {
        const uint64_t keep = policy_evict_last(), once = P.tiles_n > 1 || P.tiles_m > 1 ? policy_normal() : policy_evict_first();
        SgRing ring(S), sets(nres ? nres : 1);  // slices; sets of resident weights
        int held_g = -1, held_n = -1;
        const uint32_t a_box = MODE == SG_DW ? SG_A_BYTES : (uint32_t)P.a_rows * 128u;
        constexpr int STEP = MODE == SG_I8 ? 128 : 64;  // elements of 128 bytes
        auto load_b = [&](uint32_t to, int j, int g, int nb, uint32_t bar) {
            if constexpr (MODE == SG_Y) {
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    if (h * 64 < bn) sg_load(to + (uint32_t)h * 8192u, &mapB, nb * bn + h * 64, j * 64, g, bar, keep);
            } else {
                sg_load(to, &mapB, j * STEP, nb * bn, g, bar, keep);
            }
        };
        walk([&](const SegRows& t, int mb, int nb, int64_t) {
            const int slices = slices_of(t);
            if (MODE != SG_DW && nres && (t.g != held_g || nb != held_n)) {
                if (!sg_wait(b_empty(sets.s), sets.parity ^ 1u)) { failed = true; return false; }
                sg_expect(b_full(sets.s), b_tile);
                for (int j = 0; j < slices; ++j) load_b(res0 + sets.s * b_tile + (uint32_t)j * b_bytes, j, t.g, nb, b_full(sets.s));
                sets.next();
                held_g = t.g;
                held_n = nb;
            }
            for (int j = 0; j < slices; ++j, ring.next()) {
                const int s = (int)ring.s;
                if (!sg_wait(empty(s), ring.parity ^ 1u)) { failed = true; return false; }
                const bool both = pair && t.hi - t.lo > TC_ROWS;
                sg_expect(full(s), (both ? 2 * a_box : a_box) + (nres ? 0u : b_bytes));
                const uint32_t a0 = ring0 + (uint32_t)s * slot_bytes, b0 = a0 + a_bytes;
                if constexpr (MODE == SG_DW) {
                    const int row = (int)(t.lo + (int64_t)j * 64);
#pragma unroll
                    for (int h = 0; h < 2; ++h) sg_load(a0 + (uint32_t)h * 8192u, &mapA, mb * 128 + h * 64, row, 0, full(s), once);
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (h * 64 < bn) sg_load(b0 + (uint32_t)h * 8192u, &mapB, nb * bn + h * 64, row, 0, full(s), once);
                } else {
                    sg_load(a0, &mapA, j * STEP, (int)t.lo, 0, full(s), once);
                    if (both) sg_load(a0 + SG_A_BYTES, &mapA, j * STEP, (int)t.lo + TC_ROWS, 0, full(s), once);
                    if (!nres) load_b(b0, j, t.g, nb, full(s));
                }
            }
            return true;
        });
        if (failed && lane == 0) {
            // do not leave while copies into this CTA's shared memory may still be in flight
            ring.drain([&](uint32_t q) { return full((int)q); });
            sets.drain([&](uint32_t q) { return b_full(q); });
        }
    } else if (warp == 1) {
        const uint32_t idesc = MODE == SG_I8 ? make_idesc_i8(bn) : make_idesc(bn, MODE != SG_DX, MODE == SG_DW);
        SgRing ring(S), sets(nres ? nres : 1);
        uint32_t lt = 0, second = 0, res = 0, last_set = 0;  // tiles; tiles with a second half
        int held_g = -1, held_n = -1;
        walk([&](const SegRows& t, int, int nb, int64_t) {
            if (nres && (t.g != held_g || nb != held_n)) {
                if (sets.uses > 0) sg_commit(b_empty(last_set));  // the products of the last set are done
                if (!sg_wait(b_full(sets.s), sets.parity)) { failed = true; return false; }
                last_set = sets.s;
                res = res0 + last_set * b_tile;
                sets.next();
                held_g = t.g;
                held_n = nb;
            }
            const bool both = pair && t.hi - t.lo > TC_ROWS;
            const uint32_t a = pair ? 0u : lt & 1u;
            const uint32_t dacc = tmem_base + a * acc_cols;
            const int slices = slices_of(t);
            if (!sg_wait(acc_empty(a), ((pair ? lt : lt >> 1) & 1u) ^ 1u) || (both && !sg_wait(acc_empty(1), (second & 1u) ^ 1u))) { failed = true; return false; }
            for (int j = 0; j < slices; ++j, ring.next()) {
                const int s = (int)ring.s;
                const uint32_t a0 = ring0 + (uint32_t)s * slot_bytes, b0 = nres ? res + (uint32_t)j * b_bytes : a0 + a_bytes;
                if (!sg_wait(full(s), ring.parity)) { failed = true; return false; }
                if constexpr (MODE == SG_DW) {
                    const int have = (int)(t.hi - t.lo - (int64_t)j * 64);
                    if (have < 64) {  // rows of the next segment: 128 bytes each, from `have` to the end of every box
                        for (int box = 0; box < 2 + bn / 64; ++box)
                            for (uint32_t o = (uint32_t)have * 128u + (uint32_t)lane * 16u; o < 8192u; o += 512u)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a0 + (uint32_t)box * 8192u + o), "r"(0u) : "memory");
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                }
                tc_fence_after();
                // K-major: rows 128 bytes apart, groups of 8 rows 1024, a k-step 32 bytes along the row.  MN-major: 16
                // contraction rows of 128 bytes a k-step, boxes of 64 columns 8192 bytes apart.  A k-step adds a constant to
                // the descriptors' address field (units of 16 bytes)
                constexpr bool A_MN = MODE == SG_DW, B_MN = MODE == SG_DW || MODE == SG_Y;
                const uint64_t ad = make_smem_desc(a0, A_MN ? 8192 : 16, 1024, SG_SW128), bd = make_smem_desc(b0, B_MN ? 8192 : 16, 1024, SG_SW128);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    const uint64_t da = ad + (uint64_t)(kk * (A_MN ? 128 : 2)), db = bd + (uint64_t)(kk * (B_MN ? 128 : 2));
                    const uint32_t more = kk > 0 ? 1u : j > 0;
                    if constexpr (MODE == SG_I8) sg_mma_i8(dacc, da, db, idesc, more);
                    else sg_mma_bf16(dacc, da, db, idesc, more);
                }
                if (MODE != SG_DW && both) {
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) {
                        const uint64_t da = ad + (uint64_t)(SG_A_BYTES / 16 + kk * 2), db = bd + (uint64_t)(kk * (B_MN ? 128 : 2));
                        const uint32_t more = kk > 0 ? 1u : j > 0;
                        if constexpr (MODE == SG_I8) sg_mma_i8(dacc + acc_cols, da, db, idesc, more);
                        else sg_mma_bf16(dacc + acc_cols, da, db, idesc, more);
                    }
                }
                sg_commit(empty(s));
            }
            sg_commit(acc_full(a));
            if (both) {
                sg_commit(acc_full(1));
                ++second;
            }
            ++lt;
            return true;
        });
        // every commit has arrived before the CTA leaves (those of resident weights before later ones of the ring)
        if (lane == 0) ring.drain([&](uint32_t q) { return empty((int)q); });
    } else {
        const int ew = warp - 2, quarter = warp & 3, sub = ew >> 2;  // tensor-memory lanes 32 * (warp % 4)..: hardware rule
        const uint32_t stg = stage0 + (uint32_t)ew * SG_STAGING;
        const uint32_t floor = P.relu ? 0u : 0xFF80FF80u;
        uint32_t lt = 0, second = 0, met = 0;
        int staged_g = -1, staged_n = -1;
        walk([&](const SegRows& t, int mb, int nb, int64_t part) {
            if ((MODE == SG_Y || MODE == SG_I8) && (t.g != staged_g || nb != staged_n)) {  // the same in all epilogue warps
                const int c = tid - 64, col = nb * bn + c;
                if (!sg_meet(meet, met++)) { failed = true; return false; }
                if (c < 256) {
                    s_cols[0][c] = P.bias && c < bn && col < P.cols_out ? P.bias[(int64_t)t.g * P.cols_out + col] : 0.f;
                    if constexpr (MODE == SG_I8) s_cols[1][c] = c < bn && col < P.cols_out ? P.sw[col] : 0.f;
                }
                if (!sg_meet(meet, met++)) { failed = true; return false; }
                staged_g = t.g;
                staged_n = nb;
            }
            const int halves = pair && t.hi - t.lo > TC_ROWS ? 2 : 1;
            for (int half = 0; half < halves; ++half) {
                const uint32_t a = pair ? (uint32_t)half : lt & 1u;
                const int64_t row0 = t.lo + half * TC_ROWS + quarter * 32;  // (not SG_DW)
                const int64_t left = MODE == SG_DW ? (int64_t)P.rows_out - mb * 128 - quarter * 32 : t.hi - row0;
                const int rows = (int)(left < 32 ? left : 32);
                float sx = 0.f;
                if (MODE == SG_I8 && lane < rows) sx = P.sx[row0 + lane];
                if (!sg_wait(acc_full(a), (half ? second : pair ? lt : lt >> 1) & 1u)) { failed = true; return false; }
                tc_fence_after();
                const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + a * acc_cols;
                const bool cut = MODE == SG_DW && (t.a != t.lo || t.b != t.hi);
                const int c_base = nb * bn, c_end = P.cols_out;
                // four sums at column c of the tile -> values before relu
                auto finish4 = [&](int c, const uint32_t* r, float* f) {
                    if constexpr (MODE == SG_I8) {
                        const float4 w = *reinterpret_cast<const float4*>(&s_cols[1][c]), b = *reinterpret_cast<const float4*>(&s_cols[0][c]);
                        const float wv[4] = {w.x, w.y, w.z, w.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) f[q] = sg_i8_value((int)r[q], sx, wv[q], bv[q]);  // (zeros where there is no bias)
                    } else if constexpr (MODE == SG_Y) {
                        const float4 b = *reinterpret_cast<const float4*>(&s_cols[0][c]);
                        f[0] = __uint_as_float(r[0]) + b.x; f[1] = __uint_as_float(r[1]) + b.y; f[2] = __uint_as_float(r[2]) + b.z; f[3] = __uint_as_float(r[3]) + b.w;
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) f[q] = __uint_as_float(r[q]);
                    }
                };
                auto send = [&](auto* out, int64_t ld, bool vec, bool bulk, int y) {
                    using O = typename std::remove_pointer<decltype(out)>::type;
                    constexpr int WIDE = 64 / sizeof(O), PER = Chunk<O>::N;  // columns of a staging row: 16 or 32; of a chunk
                    for (int cb = sub; cb * WIDE < bn; cb += SG_EPI_WARPS / 4) {
                        if (c_base + cb * WIDE >= c_end || rows <= 0) break;  // the whole warp
                        uint32_t r[WIDE];
#pragma unroll
                        for (int h = 0; h < WIDE / 16; ++h) tmem_ld16(taddr + (uint32_t)(cb * WIDE + h * 16), r + h * 16);
                        tmem_ld_wait();
                        float f[WIDE];
                        sg_staging_free(lane);
#pragma unroll
                        for (int q = 0; q < WIDE / PER; ++q) {
#pragma unroll
                            for (int k = 0; k < PER; k += 4) finish4(cb * WIDE + q * PER + k, r + q * PER + k, f + q * PER + k);
                            sg_stage(stg, lane, q, MODE == SG_DW || MODE == SG_DX ? Chunk<O>::pack(f + q * PER) : sg_pack(f + q * PER, (O*)nullptr, floor));
                        }
                        if (bulk && rows == 32) {
                            sg_box_out(stg, &mapO, c_base + cb * WIDE, y, lane);
                        } else {
                            __syncwarp();
                            sg_rows_out<O>(stg, out, ld, rows, c_base + cb * WIDE, c_end, vec, lane);
                        }
                    }
                };
                if constexpr (MODE == SG_DW) {
                    const int64_t off = (int64_t)(mb * 128 + quarter * 32) * P.cols_out;
                    const int64_t size = (int64_t)P.rows_out * P.cols_out;
                    if (cut) {
                        // cut at the part's start: partial 2p, else (at its end) 2p + 1
                        const int64_t which = 2 * part + (t.a >= part * P.part_rows ? 1 : 0);
                        send(P.part + which * size + off, P.cols_out, P.cols_out % 4 == 0, P.bulk != 0, (int)(which * P.rows_out) + mb * 128 + quarter * 32);
                    } else {
                        send((T*)P.out + t.g * size + off, P.cols_out, P.vec != 0, false, 0);
                    }
                } else {
                    send((T*)P.out + row0 * P.cols_out, P.cols_out, P.vec != 0, P.bulk != 0, (int)row0);
                    // rare: such rows once more, element by element, behind their stores (asked before send, where the scale has just been
                    // loaded, 170k x 256 -> 256 took 1 us longer; as a choice for each sum 5 us)
                    if (MODE == SG_I8 && __any_sync(0xFFFFFFFFu, sg_i8_wide(sx))) {
                        sg_stores_done(lane);
                        __syncwarp();
                        T* const out = (T*)P.out + (row0 + lane) * P.cols_out + c_base;
                        constexpr int WIDE = 64 / sizeof(T), EVERY = SG_EPI_WARPS / 4;  // the columns that this warp has stored, 16 at a time
                        for (int i = 0;; ++i) {
                            const int c0 = (sub + i / (WIDE / 16) * EVERY) * WIDE + i % (WIDE / 16) * 16;
                            if (c0 >= bn || c_base + c0 >= c_end) break;
                            uint32_t r[16];
                            tmem_ld16(taddr + (uint32_t)c0, r);
                            tmem_ld_wait();
#pragma unroll
                            for (int q = 0; q < 16; ++q) {
                                float v = sg_i8_wide_value((int)r[q], sx, s_cols[MODE == SG_I8 ? 1 : 0][c0 + q], s_cols[0][c0 + q]);
                                asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(__uint_as_float(floor & 0xFFFF0000u)));
                                if (sg_i8_wide(sx) && lane < rows && c_base + c0 + q < c_end) out[c0 + q] = T(v);
                            }
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(acc_empty(a));
                second += (uint32_t)half;
            }
            ++lt;
            return true;
        });
        sg_stores_done(lane);
        if (MODE == SG_Y || MODE == SG_DX) sg_zero_outside<SG_EPI_WARPS>(P, (T*)P.out);
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
// what sg_box_out stores through: rows on 16 bytes
bool make_map_rows_out(CUtensorMap* m, void* ptr, int type, int64_t rows, int64_t cols);
bool tensor_map_encoder_available();
// SG_Y, SG_DX or SG_DW of fp32 (segment_gemm_f32.cu); slot: of allow_big_smem
gnn_status segment_gemm_f32(const char* who, int mode, int slot, const CUtensorMap& mapA, const CUtensorMap& mapB, SegGemmParams& P, int64_t part_rows_all, cudaStream_t st);
// the output's map, or that of the partials (SG_DW); other is passed in its place where rows do not start on 16 bytes
inline bool sg_out_map(CUtensorMap* m, const CUtensorMap& other, SegGemmParams& P, void* ptr, int type, int64_t rows) {
    P.bulk = (size_t)P.cols_out * (type == 0 ? 2 : 4) % 16 == 0;
    *m = other;
    return !P.bulk || make_map_rows_out(m, ptr, type, rows, P.cols_out);
}

// output columns of a tile: as few blocks of at most `most` as cover them, evened out, in steps of 64; halved while there are
// fewer tiles than SMs (a tile's weights then arrive through more SMs)
inline int sg_block(int cols, int most, int64_t row_tiles) {
    const int blocks = (cols + most - 1) / most;
    int bn = ((cols + blocks - 1) / blocks + 63) / 64 * 64;
    while (bn > 64 && row_tiles * ((cols + bn - 1) / bn) < 148) bn = (bn / 2 + 63) / 64 * 64;
    return bn;
}

// How the tiles of SG_Y, SG_DX and SG_I8 are dealt out (see above).  Pairs: where the weights of a tile are too many to stay, contractions of
// eight slices and a tile of 256 rows for every SM (65,536 x 1024 -> 1024 over 64 segments: 144 us in ones, 138 in pairs, both with stores by the warps).
// In pairs / in ones, short runs: 65,536 rows of 4 types 512 x 1024 73 / 94 us, 1024 x 1024 119 / 150, 768 x 768 79 / 88; 40,000 rows of 8 types 512 x 512 29.6 / 29.1.
// Otherwise ranges where all weights together are a fraction of L2 and the rows give every SM a few tiles.  Ranges / tiles dealt out, 128 x 128 bf16: 38,000
// rows of 4 types 9.1 / 9.8 us, 170,000 rows of 12 types 18.1 / 24.4, of 330 22.3 / 30.5; fewer tiles than that: 30,000 rows 8.1 / 8.1, 10,000 7.6 / 7.1;
// weights over 32 MB make no difference (100,000 rows of 190 types 512 x 256: 45 / 45).  (700 types, 243 rows each: 25.0 / 31.0, where the rule deals out.)
inline bool sg_stays(const SegGemmParams& P) { return SG_EPI_WARPS * SG_STAGING + (size_t)P.bn * 128 * P.slices + 4 * SG_A_BYTES <= SG_SMEM_MAX; }
inline void sg_deal(SegGemmParams& P, size_t weight_bytes, bool pairs = true) {
    const int64_t row_tiles = P.N / TC_ROWS + P.G;
    P.pair = pairs && !sg_stays(P) && P.slices >= 8 && P.N / (2 * TC_ROWS) * P.tiles_n >= 148;
    P.ranges = !P.pair && weight_bytes <= ((size_t)32 << 20) && P.N / TC_ROWS * P.tiles_n >= 296 && P.G <= P.N / 512 && P.tiles_n <= 148 ? 148 / P.tiles_n : 0;
    P.units = (P.ranges ? P.ranges : P.pair ? P.N / (2 * TC_ROWS) + P.G : row_tiles) * P.tiles_n;
    if (P.ranges) {
        const int64_t blocks = (P.N >> 5) + P.G;
        P.per_range = (unsigned)(blocks / P.ranges);
        P.longer = (unsigned)(blocks % P.ranges);
    }
}

template <int MODE, typename T>
static gnn_status sg_launch(const char* who, int which, const CUtensorMap& mapA, const CUtensorMap& mapB, SegGemmParams& P, int64_t part_rows_all, cudaStream_t st) {
    const auto kernel = segment_gemm_kernel<MODE, T>;
    CUtensorMap mapO;
    if (MODE == SG_DW ? !sg_out_map(&mapO, mapA, P, P.part, 2, part_rows_all) : !sg_out_map(&mapO, mapA, P, P.out, sizeof(T) == 2 ? 0 : 2, P.N))
        GNN_FAIL(GNN_ERR_CUDA, "%s: tensor map encoding failed", who);
    const gnn_status rc = allow_big_smem(who, (const void*)kernel, which, SG_SMEM_MAX);
    if (rc != GNN_OK) return rc;
    const size_t fixed = SG_EPI_WARPS * SG_STAGING, b_bytes = (size_t)P.bn * 128, tile = MODE == SG_DW ? 0 : b_bytes * P.slices;
    // resident weights: two sets where they leave the ring eight slots, one where they leave it four
    P.resident = MODE != SG_DW && P.ranges > 0 ? (fixed + 2 * tile + 8 * SG_A_BYTES <= SG_SMEM_MAX ? 2 : fixed + tile + 4 * SG_A_BYTES <= SG_SMEM_MAX ? 1 : 0) : 0;
    const size_t slot = (P.pair ? 2 : 1) * SG_A_BYTES + (P.resident ? 0 : b_bytes), held = (size_t)P.resident * tile;
    int stages = (int)((SG_SMEM_MAX - fixed - held) / slot);
    P.stages = stages > SG_MAX_STAGES ? SG_MAX_STAGES : stages;
    int cols = 32;
    while (cols < 2 * P.bn) cols <<= 1;
    P.tmem_cols = cols;
    launch_overlapped(kernel, dim3((unsigned)(P.units < 148 ? P.units : 148)), dim3(SG_THREADS), fixed + held + (size_t)P.stages * slot, st, mapA, mapB, mapO, P);
    GNN_CHECK_LAUNCH(who);
    return GNN_OK;
}

}  // namespace gnn
