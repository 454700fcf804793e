// The products of segment_gemm.cuh in fp32, on the bf16 tensor cores: every value is split exactly into three bf16 terms
// (x = x1 + x2 + x3) and the six products of terms with i + j <= 4 are added, by size: x1 y1; x1 y2 + x2 y1; x1 y3 + x2 y2 +
// x3 y1.  The three sums have accumulators of their own side by side: tensor-core sums cut off what lies under the last bit of a
// 24-bit sum, which costs least where products meet only those of their size; and the levels of B side by side are one operand
// three times as wide, so that a k-step is three MMAs (x1 with all levels, x2 with two, x3 with one; four for 128 columns,
// which pass the 256 of an MMA) where products one by one are six.
//
// The rows are split on the way: converter warps read fp32 slices of 32 contraction elements from shared memory and write the
// three levels into tensor memory, which the MMAs read as A (SG_DW: X transposed, a feature per lane).  Two groups of four warps
// take slices in turn, so that one slice's chain (wait, read, split, write, arrive) runs beside the other's.  The weights' levels are
// written once per call by split_rows_kernel (SG_Y, SG_DX); dY's levels (SG_DW) go to shared memory, rows of 128 bytes as the
// copy engine would lay them.  Rows of the next segment at the end of a segment's last slice (SG_DW) become zeros while they are
// split.  Only the loader and the epilogue look segments up: what a slice is goes with it from the loader to the converters and
// from them to the MMA issuer.
// Splitting in a pass of its own (all operands as planes in memory): 170,000 x 100 -> 47 over 7 segments 74 us, gradients of
// 40,000 x 128 x 64 70 us; this kernel 35 and 31 us.  A slice takes 1250 cycles, its MMAs alone 384: what bounds it is the chain of
// waits, issue and commits of the MMA issuer beside the other warps' work (MMAs in another order, the split done before the wait for its
// operand buffer: no change).
//
//   warp 0       loader: fp32 slices of the rows (32 contraction elements x 128 rows; SG_DW: 32 rows of 128 features and of bn
//                columns), the weights' levels, 64 deep, in a ring of their own
//   warp 1       MMA issuer
//   warps 2-9    epilogue: the accumulators added, then as in segment_gemm.cuh
//   warps 10-17  converters
#include "segment_gemm.cuh"

namespace gnn {

constexpr int SF_EPI_WARPS = 8, SF_CONV_WARPS = 8, SF_GROUPS = 2, SF_GROUP_WARPS = SF_CONV_WARPS / SF_GROUPS;
constexpr int SF_THREADS = 32 * (2 + SF_EPI_WARPS + SF_CONV_WARPS);
constexpr int SF_RAW_SLOTS = 6, SF_B_SLOTS = 4;  // at most
constexpr int SF_SLICE = 32;                     // contraction elements of a slice
constexpr uint32_t SF_OP_LEVEL = SF_SLICE / 2, SF_OP_COLS = 3 * SF_OP_LEVEL;  // tensor-memory columns of a level, of a slice of A
// what a slice is: its contraction elements that exist, and
constexpr uint32_t SF_LAST = 1u << 8, SF_END = 1u << 9;  // the last of its tile; nothing: the work is done

struct SegGemmF32Layout {
    int raw_slots, b_slots;  // ring slots; b_slots: of the weights' levels (SG_DW: of dY's, one per group)
    uint32_t raw_bytes, b_bytes;
    int acc_bufs;
};

// 8 fp32 values -> their three bf16 terms, 16 bytes each
__device__ __forceinline__ void sf_split(float* x, uint4* level) {
#pragma unroll
    for (int l = 0; l < 3; ++l) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            w[j / 2] = Chunk<__nv_bfloat16>::pack2(x[j], x[j + 1]);
            if (l < 2) {  // exact: the rounded term shares the leading bits
                x[j] -= __uint_as_float(w[j / 2] << 16);
                x[j + 1] -= __uint_as_float(w[j / 2] & 0xFFFF0000u);
            }
        }
        level[l] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ __forceinline__ void sf_read16(uint32_t addr, float* f) {
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]) : "r"(addr) : "memory");
}

// 16 columns of this warp's 32 lanes of tensor memory
__device__ __forceinline__ void sf_tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
// 32 values of a row (or of a feature down the rows) -> three levels of 16 columns
__device__ __forceinline__ void sf_split32(float* x, uint32_t to) {
    uint32_t w[3][16];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint4 lv[3];
        sf_split(x + 8 * c, lv);
#pragma unroll
        for (int l = 0; l < 3; ++l) { w[l][4 * c] = lv[l].x; w[l][4 * c + 1] = lv[l].y; w[l][4 * c + 2] = lv[l].z; w[l][4 * c + 3] = lv[l].w; }
    }
#pragma unroll
    for (int l = 0; l < 3; ++l) sf_tmem_st16(to + (uint32_t)l * SF_OP_LEVEL, w[l]);
}

template <int MODE>
__global__ void __launch_bounds__(SF_THREADS, 1)
segment_gemm_f32_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ CUtensorMap mapO,
                        const SegGemmParams P, const SegGemmF32Layout L) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    // r_full, r_empty [raw], b_full, b_empty [b], o_full, o_empty [groups], acc_full, acc_empty [2], meet
    __shared__ __align__(8) uint64_t bars[2 * SF_RAW_SLOTS + 2 * SF_B_SLOTS + 2 * SF_GROUPS + 5];
    __shared__ __align__(16) float s_bias[128];
    __shared__ uint32_t tmem_base_slot, s_raw[SF_RAW_SLOTS], s_op[SF_GROUPS];  // what the slice of a slot, of an operand buffer is
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int bn = P.bn;
    const uint32_t base = smem_u32(smem_raw);
    if (base & 1023u) {  // (never: the array's own alignment)
        if (tid == 0) atomicExch(P.status, 7);
        return;
    }
    const uint32_t raw0 = base, b0 = raw0 + (uint32_t)L.raw_slots * L.raw_bytes, stage0 = b0 + (uint32_t)L.b_slots * L.b_bytes;
    const uint32_t b_level = L.b_bytes / 3;
    const uint32_t bar0 = smem_u32(bars);
    auto r_full = [&](uint32_t s) { return bar0 + 8u * s; };
    auto r_empty = [&](uint32_t s) { return bar0 + 8u * (SF_RAW_SLOTS + s); };
    auto b_full = [&](uint32_t s) { return bar0 + 8u * (2 * SF_RAW_SLOTS + s); };
    auto b_empty = [&](uint32_t s) { return bar0 + 8u * (2 * SF_RAW_SLOTS + SF_B_SLOTS + s); };
    auto o_full = [&](uint32_t o) { return bar0 + 8u * (2 * SF_RAW_SLOTS + 2 * SF_B_SLOTS + o); };
    auto o_empty = [&](uint32_t o) { return bar0 + 8u * (2 * SF_RAW_SLOTS + 2 * SF_B_SLOTS + SF_GROUPS + o); };
    auto acc_full = [&](uint32_t a) { return bar0 + 8u * (2 * SF_RAW_SLOTS + 2 * SF_B_SLOTS + 2 * SF_GROUPS + a); };
    auto acc_empty = [&](uint32_t a) { return bar0 + 8u * (2 * SF_RAW_SLOTS + 2 * SF_B_SLOTS + 2 * SF_GROUPS + 2 + a); };
    const uint32_t meet = bar0 + 8u * (2 * SF_RAW_SLOTS + 2 * SF_B_SLOTS + 2 * SF_GROUPS + 4);
    const uint32_t nraw = (uint32_t)L.raw_slots, nb_slots = (uint32_t)L.b_slots, nacc = (uint32_t)L.acc_bufs;

    if (tid == 0) {
        for (uint32_t s = 0; s < nraw; ++s) { mbar_init(r_full(s), 1); mbar_init(r_empty(s), SF_GROUP_WARPS); }
        for (uint32_t s = 0; s < nb_slots; ++s) { mbar_init(b_full(s), 1); mbar_init(b_empty(s), 1); }
        for (uint32_t o = 0; o < SF_GROUPS; ++o) { mbar_init(o_full(o), SF_GROUP_WARPS); mbar_init(o_empty(o), 1); }
        for (uint32_t a = 0; a < 2; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), SF_EPI_WARPS); }
        mbar_init(meet, SF_EPI_WARPS);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapA)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapB)) : "memory");
    }
    sg_touch(P);
    if (warp == 1) tmem_alloc(smem_u32(&tmem_base_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait_exclusive();  // (set up early, the next kernel's blocks cost these more than its start saves: dW 36 -> 39 us)
    if (P.reset && blockIdx.x == 0 && tid == 0) *P.status = 0;
    const uint32_t tmem_base = tmem_base_slot;
    const uint32_t acc_cols = 3u * (uint32_t)bn;  // one accumulator per size of the products
    const uint32_t op0 = tmem_base + nacc * acc_cols;
    bool failed = false;
    const bool two_acc = nacc == 2;

    if (warp == 0) {
        const uint64_t keep = policy_evict_last(), once = P.tiles_n > 1 || P.tiles_m > 1 ? policy_normal() : policy_evict_first();
        SgRing raw((int)nraw), ws((int)nb_slots);
        sg_walk<MODE>(P, [&](const SegRows& t, int mb, int nb, int64_t) {
            const int length = MODE == SG_DW ? (int)(t.hi - t.lo) : P.contraction;
            for (int k = 0; k < length; k += SF_SLICE) {
                const uint32_t s = raw.s, to = raw0 + s * L.raw_bytes;
                if (!sg_wait(r_empty(s), raw.parity ^ 1u)) { failed = true; return false; }
                const int have = length - k;
                s_raw[s] = have > SF_SLICE ? (uint32_t)SF_SLICE : (uint32_t)have | SF_LAST;  // all lanes: the one that arrives too
                if constexpr (MODE == SG_DW) {  // boxes of 32 rows x 32 columns
                    sg_expect(r_full(s), (uint32_t)(4 + bn / 32) * 4096u);
                    const int row = (int)(t.lo + k);
#pragma unroll
                    for (int h = 0; h < 4; ++h) sg_load(to + (uint32_t)h * 4096u, &mapA, mb * 128 + h * 32, row, 0, r_full(s), once);
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (h * 32 < bn) sg_load(to + (uint32_t)(4 + h) * 4096u, &mapB, nb * bn + h * 32, row, 0, r_full(s), once);
                } else {
                    sg_expect(r_full(s), (uint32_t)P.a_rows * 128u);
                    sg_load(to, &mapA, k, (int)t.lo, 0, r_full(s), once);
                    if ((k & 32) == 0) {  // the weights' levels for this slice and the next
                        const uint32_t q = ws.s;
                        if (!sg_wait(b_empty(q), ws.parity ^ 1u)) { failed = true; raw.next(); return false; }
                        sg_expect(b_full(q), L.b_bytes);
                        const uint32_t bs = b0 + q * L.b_bytes;
#pragma unroll
                        for (int l = 0; l < 3; ++l) {
                            if constexpr (MODE == SG_Y) {
#pragma unroll
                                for (int h = 0; h < 2; ++h)
                                    if (h * 64 < bn) sg_load(bs + (uint32_t)l * b_level + (uint32_t)h * 8192u, &mapB, nb * bn + h * 64, k, l * P.G + t.g, b_full(q), keep);
                            } else {
                                sg_load(bs + (uint32_t)l * b_level, &mapB, k, nb * bn, l * P.G + t.g, b_full(q), keep);
                            }
                        }
                        ws.next();
                    }
                }
                raw.next();
            }
            return true;
        });
        for (int e = 0; e < SF_GROUPS && !failed; ++e, raw.next()) {  // the end, to each group
            if (!sg_wait(r_empty(raw.s), raw.parity ^ 1u)) { failed = true; break; }
            s_raw[raw.s] = SF_END;
            sg_expect(r_full(raw.s), 0);
        }
        if (failed && lane == 0) {
            // do not leave while copies into this CTA's shared memory may still be in flight
            raw.drain(r_full);
            if (MODE != SG_DW) ws.drain(b_full);
        }
    } else if (warp == 1) {
        constexpr int B_MN = MODE != SG_DX;
        const uint32_t wide = make_idesc(bn == 64 ? 192 : 256, B_MN), two = make_idesc(2 * bn, B_MN), one = make_idesc(bn, B_MN);
        SgRing ws((int)nb_slots);
        uint32_t it = 0, lt = 0;
        bool first = true;  // slice of its tile
        int k = 0;          // slices of the tile so far
        while (true) {
            const uint32_t o = it % SF_GROUPS, a = two_acc ? lt & 1u : 0u, d0 = tmem_base + a * acc_cols;
            if (!sg_wait(o_full(o), (it / SF_GROUPS) & 1u)) { failed = true; break; }
            const uint32_t info = s_op[o];
            ++it;
            if (info & SF_END) break;
            if (first && !sg_wait(acc_empty(a), ((two_acc ? lt >> 1 : lt) & 1u) ^ 1u)) { failed = true; break; }
            const uint32_t q = MODE == SG_DW ? o : ws.s;
            if (MODE != SG_DW && (k & 1) == 0 && !sg_wait(b_full(q), ws.parity)) { failed = true; break; }
            tc_fence_after();
            const uint32_t at = op0 + o * SF_OP_COLS;
            // MN-major: boxes of 64 columns, 64 contraction rows of 128 bytes each (SG_DW: 32); K-major: rows of 64.  Levels and
            // k-steps add to the descriptor's address field (units of 16 bytes); levels lie one after the other, as columns do
            constexpr uint32_t STEP = MODE == SG_DX ? 2 : 128;
            const uint64_t bd = make_smem_desc(b0 + q * L.b_bytes, MODE == SG_DX ? 16 : MODE == SG_DW ? 4096 : 8192, 1024, SG_SW128) + (MODE == SG_DW ? 0u : (uint32_t)(k & 1) * 2u * STEP);
            const uint64_t third = bd + 2 * (b_level / 16);
            const int steps = (int)((info & 255u) + 15u) / 16;
#pragma unroll
            for (int kk = 0; kk < SF_SLICE / 16; ++kk) {
                if (kk >= steps) break;
                const uint32_t more = kk > 0 ? 1u : first ? 0u : 1u, x1 = at + (uint32_t)kk * 8u;
                sg_mma_bf16_ts(d0, x1, bd + kk * STEP, wide, more);
                if (bn == 128) sg_mma_bf16_ts(d0 + 256, x1, third + kk * STEP, one, more);
                sg_mma_bf16_ts(d0 + (uint32_t)bn, x1 + SF_OP_LEVEL, bd + kk * STEP, two, 1u);
                sg_mma_bf16_ts(d0 + 2u * (uint32_t)bn, x1 + 2 * SF_OP_LEVEL, bd + kk * STEP, one, 1u);
            }
            sg_commit(o_empty(o));
            const bool last = (info & SF_LAST) != 0;
            if (MODE != SG_DW && ((k & 1) || last)) {
                sg_commit(b_empty(q));
                ws.next();
            }
            ++k;
            first = last;
            if (last) {
                sg_commit(acc_full(a));
                ++lt;
                k = 0;
            }
        }
        // every commit has arrived before the CTA leaves (the end used an operand buffer without one)
        if (lane == 0 && !failed) {
            --it;
            for (uint32_t i = it > SF_GROUPS ? it - SF_GROUPS : 0u; i < it; ++i) mbar_wait_bounded(o_empty(i % SF_GROUPS), (i / SF_GROUPS) & 1u);
            if (MODE != SG_DW) ws.drain(b_empty);
        }
    } else if (warp >= 2 + SF_EPI_WARPS) {
        const uint32_t grp = (uint32_t)(warp - 2 - SF_EPI_WARPS) / SF_GROUP_WARPS;
        const int quarter = warp & 3;  // a warp reaches the 32 lanes of tensor memory of its number modulo 4
        SgRing raw((int)nraw);
        if (grp == 1) raw.next();
        for (uint32_t turn = 0;; ++turn) {
            const uint32_t s = raw.s;
            if (!sg_wait(r_full(s), raw.parity) || !sg_wait(o_empty(grp), (turn & 1u) ^ 1u)) { failed = true; break; }
            const uint32_t info = s_raw[s];
            const int have = (int)(info & 255u);
            if (!(info & SF_END)) {
                tc_fence_after();
                const uint32_t from = raw0 + s * L.raw_bytes;
                const uint32_t to = op0 + ((uint32_t)(quarter * 32) << 16) + grp * SF_OP_COLS;
                float x[32];
                if constexpr (MODE != SG_DW) {  // a row's 32 elements (zeros past the last: the copy engine's)
                    const uint32_t r = (uint32_t)(quarter * 32 + lane), at = from + r * 128u;
#pragma unroll
                    for (int c = 0; c < 8; ++c) sf_read16(at + (((uint32_t)c ^ (r & 7u)) << 4), x + 4 * c);
                    sf_split32(x, to);
                } else {
                    // A: feature `lane` of this quarter's box, rows down the box
                    const uint32_t box = from + (uint32_t)quarter * 4096u + (uint32_t)(lane & 3) * 4u;
#pragma unroll
                    for (int r = 0; r < 32; ++r) {
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[r]) : "r"(box + (uint32_t)r * 128u + (uint32_t)(((lane >> 2) ^ (r & 7)) << 4)) : "memory");
                        if (r >= have) x[r] = 0.f;
                    }
                    sf_split32(x, to);
                    // B: row `lane`, 8 columns at a time
                    const uint32_t bs = b0 + grp * L.b_bytes, r7 = (uint32_t)lane & 7u;
                    for (int q = warp & 3; q < bn / 8; q += SF_GROUP_WARPS) {
                        const uint32_t at = from + (uint32_t)(4 + (q >> 2)) * 4096u + (uint32_t)lane * 128u;
                        float y[8];
                        sf_read16(at + (((uint32_t)(2 * (q & 3)) ^ r7) << 4), y);
                        sf_read16(at + (((uint32_t)(2 * (q & 3) + 1) ^ r7) << 4), y + 4);
                        if (lane >= have)
#pragma unroll
                            for (int k = 0; k < 8; ++k) y[k] = 0.f;
                        uint4 lv[3];
                        sf_split(y, lv);
#pragma unroll
                        for (int l = 0; l < 3; ++l)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(bs + (uint32_t)l * b_level + (uint32_t)(q >> 3) * 4096u + (uint32_t)lane * 128u + ((((uint32_t)q & 7u) ^ r7) << 4)),
                                         "r"(lv[l].x), "r"(lv[l].y), "r"(lv[l].z), "r"(lv[l].w) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                tmem_st_wait();
                tc_fence_before();
            }
            if (lane == 0) s_op[grp] = info;
            __syncwarp();
            if (lane == 0) { mbar_arrive(r_empty(s)); mbar_arrive(o_full(grp)); }
            if (info & SF_END) break;
            raw.next();
            raw.next();
        }
    } else {
        const int ew = warp - 2, quarter = warp & 3, sub = ew >> 2;
        const uint32_t stg = stage0 + (uint32_t)ew * SG_STAGING;
        uint32_t lt = 0, met = 0;
        int staged_g = -1, staged_n = -1;
        sg_walk<MODE>(P, [&](const SegRows& t, int mb, int nb, int64_t part) {
            const uint32_t a = two_acc ? lt & 1u : 0u;
            if (MODE == SG_Y && P.bias && (t.g != staged_g || nb != staged_n)) {  // the same in all epilogue warps
                const int c = tid - 64, col = nb * bn + c;
                if (!sg_meet(meet, met++)) { failed = true; return false; }
                if (c < 128) s_bias[c] = c < bn && col < P.cols_out ? P.bias[(int64_t)t.g * P.cols_out + col] : 0.f;
                if (!sg_meet(meet, met++)) { failed = true; return false; }
                staged_g = t.g;
                staged_n = nb;
            }
            if (!sg_wait(acc_full(a), (two_acc ? lt >> 1 : lt) & 1u)) { failed = true; return false; }
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + a * acc_cols;
            const int64_t left = MODE == SG_DW ? (int64_t)P.rows_out - mb * 128 - quarter * 32 : t.hi - t.lo - quarter * 32;
            const int rows = (int)(left < 32 ? left : 32), c_base = nb * bn;
            float* out = (float*)P.out;
            bool vec = P.vec != 0, bulk = P.bulk != 0;
            int y = (int)(t.lo + quarter * 32);
            if constexpr (MODE == SG_DW) {
                const int64_t size = (int64_t)P.rows_out * P.cols_out;
                if (t.a != t.lo || t.b != t.hi) {
                    // cut at the part's start: partial 2p, else (at its end) 2p + 1
                    const int64_t which = 2 * part + (t.a >= part * P.part_rows ? 1 : 0);
                    out = P.part + which * size;
                    vec = P.cols_out % 4 == 0;
                    y = (int)(which * P.rows_out) + mb * 128 + quarter * 32;
                } else {
                    out += t.g * size;
                    bulk = false;
                }
                out += (int64_t)(mb * 128 + quarter * 32) * P.cols_out;
            } else {
                out += (t.lo + quarter * 32) * P.cols_out;
            }
            for (int cb = sub; cb * 16 < bn; cb += SF_EPI_WARPS / 4) {
                if (c_base + cb * 16 >= P.cols_out || rows <= 0) break;  // the whole warp
                uint32_t r[16], m[16], n[16];
                tmem_ld16(taddr + (uint32_t)(cb * 16), r);
                tmem_ld16(taddr + (uint32_t)(bn + cb * 16), m);
                tmem_ld16(taddr + (uint32_t)(2 * bn + cb * 16), n);
                tmem_ld_wait();
                float f[16];
#pragma unroll
                for (int q = 0; q < 16; ++q) f[q] = __uint_as_float(r[q]) + (__uint_as_float(m[q]) + __uint_as_float(n[q]));
                if (MODE == SG_Y && P.bias) {
#pragma unroll
                    for (int q = 0; q < 16; ++q) f[q] += s_bias[cb * 16 + q];
                }
                if (MODE == SG_Y && P.relu) {
#pragma unroll
                    for (int q = 0; q < 16; ++q) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(f[q]));  // NaN stays
                }
                sg_staging_free(lane);
#pragma unroll
                for (int q = 0; q < 4; ++q) sg_stage(stg, lane, q, Chunk<float>::pack(f + 4 * q));
                if (bulk && rows == 32) {
                    sg_box_out(stg, &mapO, c_base + cb * 16, y, lane);
                } else {
                    __syncwarp();
                    sg_rows_out<float>(stg, out, P.cols_out, rows, c_base + cb * 16, P.cols_out, vec, lane);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty(a));
            ++lt;
            return true;
        });
        sg_stores_done(lane);
        if (MODE != SG_DW) sg_zero_outside<SF_EPI_WARPS>(P, (float*)P.out);
    }
    if (failed) atomicExch(P.status, 7);  // GNN_ERR_TIMEOUT
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, 512);
}

template <int MODE>
static gnn_status sf_launch(const char* who, int which, const CUtensorMap& mapA, const CUtensorMap& mapB, SegGemmParams& P, int64_t part_rows_all, cudaStream_t st) {
    const auto kernel = segment_gemm_f32_kernel<MODE>;
    CUtensorMap mapO;
    if (!sg_out_map(&mapO, mapA, P, MODE == SG_DW ? (void*)P.part : P.out, 2, MODE == SG_DW ? part_rows_all : P.N)) GNN_FAIL(GNN_ERR_CUDA, "%s: tensor map encoding failed", who);
    const gnn_status rc = allow_big_smem(who, (const void*)kernel, which, SG_SMEM_MAX);
    if (rc != GNN_OK) return rc;
    const size_t fixed = SF_EPI_WARPS * SG_STAGING;
    SegGemmF32Layout L;
    // tensor memory: three accumulators of bn columns, twice where 512 columns hold them beside a slice of A per group (bn = 64)
    L.acc_bufs = 6 * P.bn + SF_GROUPS * (int)SF_OP_COLS <= 512 ? 2 : 1;
    const size_t room = SG_SMEM_MAX - fixed;
    if (MODE == SG_DW) {
        L.raw_bytes = (uint32_t)(4 + P.bn / 32) * 4096u;
        L.b_bytes = 3u * (uint32_t)(P.bn / 64) * 4096u;
        L.b_slots = SF_GROUPS;
        const size_t slots = (room - SF_GROUPS * (size_t)L.b_bytes) / L.raw_bytes;
        L.raw_slots = slots < SF_RAW_SLOTS ? (int)slots : SF_RAW_SLOTS;
    } else {
        L.raw_bytes = SG_A_BYTES;
        L.b_bytes = 3u * (uint32_t)P.bn * 128u;
        L.raw_slots = SF_RAW_SLOTS;
        const size_t slots = (room - SF_RAW_SLOTS * (size_t)L.raw_bytes) / L.b_bytes;
        L.b_slots = slots < SF_B_SLOTS ? (int)slots : SF_B_SLOTS;
    }
    launch_overlapped(kernel, dim3((unsigned)(P.units < 148 ? P.units : 148)), dim3(SF_THREADS), fixed + (size_t)L.raw_slots * L.raw_bytes + (size_t)L.b_slots * L.b_bytes, st, mapA, mapB, mapO, P, L);
    GNN_CHECK_LAUNCH(who);
    return GNN_OK;
}

gnn_status segment_gemm_f32(const char* who, int mode, int slot, const CUtensorMap& mapA, const CUtensorMap& mapB, SegGemmParams& P, int64_t part_rows_all, cudaStream_t st) {
    return mode == SG_Y ? sf_launch<SG_Y>(who, slot, mapA, mapB, P, 0, st)
         : mode == SG_DX ? sf_launch<SG_DX>(who, slot, mapA, mapB, P, 0, st) : sf_launch<SG_DW>(who, slot, mapA, mapB, P, part_rows_all, st);
}

}  // namespace gnn
