// The products of segment_gemm.cuh in fp32, on the bf16 tensor cores: every value is split exactly into three bf16 terms
// (x = x1 + x2 + x3) and the six products of terms with i + j <= 4 are added, the five small ones in an accumulator of their own:
// tensor-core sums cut off what lies under the last bit of a 24-bit sum, which costs least where the large products meet only
// one another.
//
// The rows are split on the way: converter warps read fp32 slices from shared memory and write the three levels into tensor
// memory, which the MMAs read as A (SG_DW: X transposed, a feature per lane).  Two groups of four warps take slices in turn, so
// that one slice's chain (wait, read, split, write, arrive) runs beside the other's.  The weights' levels are written once per call by
// split_rows_kernel (SG_Y, SG_DX); dY's levels (SG_DW) go to shared memory, rows of 128 bytes as the copy engine would lay
// them.  Rows of the next segment at the end of a segment's last slice (SG_DW) become zeros while they are split.
// Splitting in a pass of its own (all operands as planes in memory): 170,000 x 100 -> 47 over 7 segments 74 us, gradients of
// 40,000 x 128 x 64 70 us.
//
//   warp 0       loader: fp32 slices of the rows (64 contraction elements x 128 rows; SG_DW: 32 rows of 128 features and of bn
//                columns), the weights' levels in a ring of their own
//   warp 1       MMA issuer
//   warps 2-9    epilogue: both accumulators added, then as in segment_gemm.cuh
//   warps 10-17  converters
#include "segment_gemm.cuh"

namespace gnn {

constexpr int SF_EPI_WARPS = 8, SF_CONV_WARPS = 8, SF_GROUPS = 2, SF_GROUP_WARPS = SF_CONV_WARPS / SF_GROUPS;
constexpr int SF_THREADS = 32 * (2 + SF_EPI_WARPS + SF_CONV_WARPS);
constexpr int SF_RAW_SLOTS = 4, SF_B_SLOTS = 4;  // at most

struct SegGemmF32Layout {
    int raw_slots, b_slots;  // ring slots; b_slots: of the weights' levels (SG_DW: of dY's, one per group)
    uint32_t raw_bytes, b_bytes;
    int acc_bufs;
};

// levels of A and B of product q, small terms first: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
__device__ __forceinline__ constexpr uint32_t sf_pair_a(int q) { return q == 0 ? 2u : q == 2 || q == 3 ? 1u : 0u; }
__device__ __forceinline__ constexpr uint32_t sf_pair_b(int q) { return q == 1 ? 2u : q == 2 || q == 4 ? 1u : 0u; }

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

template <int MODE>
__global__ void __launch_bounds__(SF_THREADS, 1)
segment_gemm_f32_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const SegGemmParams P, const SegGemmF32Layout L) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    // r_full, r_empty [raw], b_full, b_empty [b], o_full, o_empty [groups], acc_full, acc_empty [2]
    __shared__ __align__(8) uint64_t bars[2 * SF_RAW_SLOTS + 2 * SF_B_SLOTS + 2 * SF_GROUPS + 4];
    __shared__ __align__(16) float s_bias[128];
    __shared__ uint32_t tmem_base_slot;
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
    const uint32_t nraw = (uint32_t)L.raw_slots, nb_slots = (uint32_t)L.b_slots, nacc = (uint32_t)L.acc_bufs;

    if (tid == 0) {
        for (uint32_t s = 0; s < nraw; ++s) { mbar_init(r_full(s), 1); mbar_init(r_empty(s), SF_GROUP_WARPS); }
        for (uint32_t s = 0; s < nb_slots; ++s) { mbar_init(b_full(s), 1); mbar_init(b_empty(s), 1); }
        for (uint32_t o = 0; o < SF_GROUPS; ++o) { mbar_init(o_full(o), SF_GROUP_WARPS); mbar_init(o_empty(o), 1); }
        for (uint32_t a = 0; a < 2; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), SF_EPI_WARPS); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapA)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapB)) : "memory");
    }
    sg_touch(P);
    if (warp == 1) tmem_alloc(smem_u32(&tmem_base_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait_exclusive();
    if (P.reset && blockIdx.x == 0 && tid == 0) *P.status = 0;
    const uint32_t tmem_base = tmem_base_slot;
    const uint32_t acc_cols = 2u * (uint32_t)bn;                  // large products, small products
    constexpr int SLICE = MODE == SG_DW ? 32 : 64;                // contraction elements
    constexpr uint32_t OP_LEVEL = SLICE / 2, OP_COLS = 3 * OP_LEVEL;  // tensor-memory columns of a level, of a slice of A
    const uint32_t op0 = tmem_base + nacc * acc_cols;
    bool failed = false;
    const bool two_acc = nacc == 2;
    auto slices_of = [&](const SegRows& t) { return MODE == SG_DW ? (int)((t.hi - t.lo + SLICE - 1) / SLICE) : P.slices; };
    // contraction elements of slice j that exist
    auto have_of = [&](const SegRows& t, int j) {
        const int64_t h = MODE == SG_DW ? t.hi - t.lo - (int64_t)j * SLICE : (int64_t)P.contraction - j * SLICE;
        return (int)(h < SLICE ? h : SLICE);
    };

    if (warp == 0) {
        const uint64_t keep = policy_evict_last(), once = P.tiles_n > 1 || P.tiles_m > 1 ? policy_normal() : policy_evict_first();
        SgRing raw((int)nraw), ws((int)nb_slots);
        sg_walk<MODE>(P, [&](const SegRows& t, int mb, int nb, int64_t) {
            const int slices = slices_of(t);
            for (int j = 0; j < slices; ++j) {
                const uint32_t s = raw.s, to = raw0 + s * L.raw_bytes;
                if (!sg_wait(r_empty(s), raw.parity ^ 1u)) { failed = true; return false; }
                if constexpr (MODE == SG_DW) {  // boxes of 32 rows x 32 columns
                    sg_expect(r_full(s), (uint32_t)(4 + bn / 32) * 4096u);
                    const int row = (int)(t.lo + (int64_t)j * SLICE);
#pragma unroll
                    for (int h = 0; h < 4; ++h) sg_load(to + (uint32_t)h * 4096u, &mapA, mb * 128 + h * 32, row, 0, r_full(s), once);
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (h * 32 < bn) sg_load(to + (uint32_t)(4 + h) * 4096u, &mapB, nb * bn + h * 32, row, 0, r_full(s), once);
                } else {  // two boxes of 32 columns, one where the contraction ends in the first
                    const bool two = have_of(t, j) > 32;
                    sg_expect(r_full(s), (uint32_t)((two ? 2 : 1) * P.a_rows) * 128u);
                    sg_load(to, &mapA, j * SLICE, (int)t.lo, 0, r_full(s), once);
                    if (two) sg_load(to + SG_A_BYTES, &mapA, j * SLICE + 32, (int)t.lo, 0, r_full(s), once);
                    const uint32_t q = ws.s;
                    if (!sg_wait(b_empty(q), ws.parity ^ 1u)) { failed = true; raw.next(); return false; }
                    sg_expect(b_full(q), L.b_bytes);
                    const uint32_t bs = b0 + q * L.b_bytes;
#pragma unroll
                    for (int l = 0; l < 3; ++l) {
                        if constexpr (MODE == SG_Y) {
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                if (h * 64 < bn) sg_load(bs + (uint32_t)l * b_level + (uint32_t)h * 8192u, &mapB, nb * bn + h * 64, j * SLICE, l * P.G + t.g, b_full(q), keep);
                        } else {
                            sg_load(bs + (uint32_t)l * b_level, &mapB, j * SLICE, nb * bn, l * P.G + t.g, b_full(q), keep);
                        }
                    }
                    ws.next();
                }
                raw.next();
            }
            return true;
        });
        if (failed && lane == 0) {
            // do not leave while copies into this CTA's shared memory may still be in flight
            raw.drain(r_full);
            if (MODE != SG_DW) ws.drain(b_full);
        }
    } else if (warp == 1) {
        const uint32_t idesc = make_idesc(bn, MODE != SG_DX, 0);
        SgRing ws((int)nb_slots);
        uint32_t it = 0, lt = 0;
        sg_walk<MODE>(P, [&](const SegRows& t, int, int, int64_t) {
            const uint32_t a = two_acc ? lt & 1u : 0u, dacc = tmem_base + a * acc_cols, small = dacc + (uint32_t)bn;
            const int slices = slices_of(t);
            if (!sg_wait(acc_empty(a), ((two_acc ? lt >> 1 : lt) & 1u) ^ 1u)) { failed = true; return false; }
            for (int j = 0; j < slices; ++j, ++it) {
                const uint32_t o = it % SF_GROUPS, q = MODE == SG_DW ? o : ws.s;
                if (!sg_wait(o_full(o), (it / SF_GROUPS) & 1u)) { failed = true; return false; }
                if (MODE != SG_DW && !sg_wait(b_full(q), ws.parity)) { failed = true; return false; }
                tc_fence_after();
                const uint32_t at = op0 + o * OP_COLS;
                // MN-major: boxes of 64 columns, SLICE contraction rows of 128 bytes each; K-major: rows of 64.  Levels and
                // k-steps add to the descriptor's address field (units of 16 bytes)
                const uint64_t bd = MODE == SG_DX ? make_smem_desc(b0 + q * L.b_bytes, 16, 1024, SG_SW128)
                                                  : make_smem_desc(b0 + q * L.b_bytes, SLICE * 128, 1024, SG_SW128);
                const uint64_t level[3] = {bd, bd + b_level / 16, bd + b_level / 8};
                const int steps = (have_of(t, j) + 15) / 16;
#pragma unroll
                for (int kk = 0; kk < SLICE / 16; ++kk) {
                    if (kk >= steps) break;
#pragma unroll
                    for (int p = 0; p < 6; ++p) {
                        const uint32_t more = kk > 0 || (p > 0 && p < 5) ? 1u : j > 0;
                        sg_mma_bf16_ts(p < 5 ? small : dacc, at + (sf_pair_a(p) * OP_LEVEL + (uint32_t)kk * 8u), level[sf_pair_b(p)] + (uint64_t)(kk * (MODE == SG_DX ? 2 : 128)), idesc, more);
                    }
                }
                sg_commit(o_empty(o));
                if (MODE != SG_DW) {
                    sg_commit(b_empty(q));
                    ws.next();
                }
            }
            sg_commit(acc_full(a));
            ++lt;
            return true;
        });
        // every commit has arrived before the CTA leaves
        if (lane == 0) {
            for (uint32_t i = it > SF_GROUPS ? it - SF_GROUPS : 0u; i < it; ++i) mbar_wait_bounded(o_empty(i % SF_GROUPS), (i / SF_GROUPS) & 1u);
            if (MODE != SG_DW) ws.drain(b_empty);
        }
    } else if (warp >= 2 + SF_EPI_WARPS) {
        const uint32_t grp = (uint32_t)(warp - 2 - SF_EPI_WARPS) / SF_GROUP_WARPS;
        const int quarter = warp & 3;  // a warp reaches the 32 lanes of tensor memory of its number modulo 4
        SgRing raw((int)nraw);
        uint32_t it = 0;
        sg_walk<MODE>(P, [&](const SegRows& t, int, int, int64_t) {
            const int slices = slices_of(t);
            for (int j = 0; j < slices; ++j, ++it, raw.next()) {
                if (it % SF_GROUPS != grp) continue;
                const uint32_t s = raw.s;
                if (!sg_wait(r_full(s), raw.parity) || !sg_wait(o_empty(grp), ((it / SF_GROUPS) & 1u) ^ 1u)) { failed = true; return false; }
                tc_fence_after();
                const uint32_t from = raw0 + s * L.raw_bytes;
                const uint32_t to = op0 + ((uint32_t)(quarter * 32) << 16) + grp * OP_COLS;
                const int have = have_of(t, j);
                if constexpr (MODE != SG_DW) {
                    const uint32_t r = (uint32_t)(quarter * 32 + lane), x7 = r & 7u;
                    // a box of 32 columns at a time: all its loads before the first split
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (h * 32 >= have) break;
                        const uint32_t at = from + (uint32_t)h * SG_A_BYTES + r * 128u;
                        float x[32];
#pragma unroll
                        for (int c = 0; c < 8; ++c) sf_read16(at + (((uint32_t)c ^ x7) << 4), x + 4 * c);
                        const int chunks = (have - h * 32 + 7) / 8;  // of 8 elements; the box is zeros past the last
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            if (c >= chunks) break;
                            uint4 lv[3];
                            sf_split(x + 8 * c, lv);
#pragma unroll
                            for (int l = 0; l < 3; ++l) tmem_st4(to + (uint32_t)l * OP_LEVEL + (uint32_t)(h * 16 + c * 4), lv[l]);
                        }
                    }
                    if (const int c = (have + 7) / 8; c & 1) {  // the second half of the last k-step: zeros
#pragma unroll
                        for (int l = 0; l < 3; ++l) tmem_st4(to + (uint32_t)l * OP_LEVEL + (uint32_t)c * 4u, make_uint4(0, 0, 0, 0));
                    }
                } else {
                    // A: feature `lane` of this quarter's box, rows down the box
                    const uint32_t box = from + (uint32_t)quarter * 4096u + (uint32_t)(lane & 3) * 4u;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float x[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int r = c * 8 + k;
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[k]) : "r"(box + (uint32_t)r * 128u + (uint32_t)(((lane >> 2) ^ k) << 4)) : "memory");
                            if (r >= have) x[k] = 0.f;
                        }
                        uint4 lv[3];
                        sf_split(x, lv);
#pragma unroll
                        for (int l = 0; l < 3; ++l) tmem_st4(to + (uint32_t)l * OP_LEVEL + (uint32_t)c * 4u, lv[l]);
                    }
                    // B: row `lane`, 8 columns at a time
                    const uint32_t bs = b0 + grp * L.b_bytes, r7 = (uint32_t)lane & 7u;
                    for (int q = warp & 3; q < bn / 8; q += SF_GROUP_WARPS) {
                        const uint32_t at = from + (uint32_t)(4 + (q >> 2)) * 4096u + (uint32_t)lane * 128u;
                        float x[8];
                        sf_read16(at + (((uint32_t)(2 * (q & 3)) ^ r7) << 4), x);
                        sf_read16(at + (((uint32_t)(2 * (q & 3) + 1) ^ r7) << 4), x + 4);
                        if (lane >= have)
#pragma unroll
                            for (int k = 0; k < 8; ++k) x[k] = 0.f;
                        uint4 lv[3];
                        sf_split(x, lv);
#pragma unroll
                        for (int l = 0; l < 3; ++l)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(bs + (uint32_t)l * b_level + (uint32_t)(q >> 3) * 4096u + (uint32_t)lane * 128u + ((((uint32_t)q & 7u) ^ r7) << 4)),
                                         "r"(lv[l].x), "r"(lv[l].y), "r"(lv[l].z), "r"(lv[l].w) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { mbar_arrive(r_empty(s)); mbar_arrive(o_full(grp)); }
            }
            return true;
        });
    } else {
        const int ew = warp - 2, quarter = warp & 3, sub = ew >> 2;
        const uint32_t stg = stage0 + (uint32_t)ew * SG_STAGING;
        uint32_t lt = 0;
        int staged_g = -1, staged_n = -1;
        sg_walk<MODE>(P, [&](const SegRows& t, int mb, int nb, int64_t part) {
            const uint32_t a = two_acc ? lt & 1u : 0u;
            if (MODE == SG_Y && P.bias && (t.g != staged_g || nb != staged_n)) {  // the same in all epilogue warps
                const int c = tid - 64, col = nb * bn + c;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (c < 128) s_bias[c] = c < bn && col < P.cols_out ? P.bias[(int64_t)t.g * P.cols_out + col] : 0.f;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                staged_g = t.g;
                staged_n = nb;
            }
            if (!sg_wait(acc_full(a), (two_acc ? lt >> 1 : lt) & 1u)) { failed = true; return false; }
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + a * acc_cols;
            const int64_t left = MODE == SG_DW ? (int64_t)P.rows_out - mb * 128 - quarter * 32 : t.hi - t.lo - quarter * 32;
            const int rows = (int)(left < 32 ? left : 32), c_base = nb * bn;
            float* out = (float*)P.out;
            bool vec = P.vec != 0;
            if constexpr (MODE == SG_DW) {
                const int64_t size = (int64_t)P.rows_out * P.cols_out;
                if (t.a != t.lo || t.b != t.hi) {
                    // cut at the part's start: partial 2p, else (at its end) 2p + 1
                    out = P.part + (2 * part + (t.a >= part * P.part_rows ? 1 : 0)) * size;
                    vec = P.cols_out % 4 == 0;
                } else {
                    out += t.g * size;
                }
                out += (int64_t)(mb * 128 + quarter * 32) * P.cols_out;
            } else {
                out += (t.lo + quarter * 32) * P.cols_out;
            }
            for (int cb = sub; cb * 16 < bn; cb += SF_EPI_WARPS / 4) {
                if (c_base + cb * 16 >= P.cols_out || rows <= 0) break;  // the whole warp
                uint32_t r[16], m[16];
                tmem_ld16(taddr + (uint32_t)(cb * 16), r);
                tmem_ld16(taddr + (uint32_t)(bn + cb * 16), m);
                tmem_ld_wait();
                float f[16];
#pragma unroll
                for (int q = 0; q < 16; ++q) f[q] = __uint_as_float(r[q]) + __uint_as_float(m[q]);
                if (MODE == SG_Y && P.bias) {
#pragma unroll
                    for (int q = 0; q < 16; ++q) f[q] += s_bias[cb * 16 + q];
                }
                if (MODE == SG_Y && P.relu) {
#pragma unroll
                    for (int q = 0; q < 16; ++q) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(f[q]));  // NaN stays
                }
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 4; ++q) sg_stage(stg, lane, q, Chunk<float>::pack(f + 4 * q));
                __syncwarp();
                sg_rows_out<float>(stg, out, P.cols_out, rows, c_base + cb * 16, P.cols_out, vec, lane);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty(a));
            ++lt;
            return true;
        });
        if (MODE != SG_DW) sg_zero_outside<SF_EPI_WARPS>(P, (float*)P.out);
    }
    if (failed) atomicExch(P.status, 7);  // GNN_ERR_TIMEOUT
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, 512);
}

template <int MODE>
static gnn_status sf_launch(const char* who, int which, const CUtensorMap& mapA, const CUtensorMap& mapB, SegGemmParams& P, cudaStream_t st) {
    const auto kernel = segment_gemm_f32_kernel<MODE>;
    const gnn_status rc = allow_big_smem(who, (const void*)kernel, which, SG_SMEM_MAX);
    if (rc != GNN_OK) return rc;
    const size_t fixed = SF_EPI_WARPS * SG_STAGING;
    SegGemmF32Layout L;
    // tensor memory: accumulators of 2 bn columns, twice where 512 columns hold them beside a slice of A per group
    constexpr int OPS = SF_GROUPS * 3 * (MODE == SG_DW ? 16 : 32);
    L.acc_bufs = 4 * P.bn + OPS <= 512 ? 2 : 1;
    if (MODE == SG_DW) {
        L.raw_bytes = (uint32_t)(4 + P.bn / 32) * 4096u;
        L.b_bytes = 3u * (uint32_t)(P.bn / 64) * 4096u;
        L.b_slots = SF_GROUPS;
        L.raw_slots = SF_RAW_SLOTS;
    } else {
        L.raw_bytes = 2 * SG_A_BYTES;
        L.b_bytes = 3u * (uint32_t)P.bn * 128u;
        L.raw_slots = 3;
        const size_t slots = (SG_SMEM_MAX - fixed - 3 * (size_t)L.raw_bytes) / L.b_bytes;
        L.b_slots = slots < SF_B_SLOTS ? (int)slots : SF_B_SLOTS;
    }
    launch_overlapped(kernel, dim3((unsigned)(P.units < 148 ? P.units : 148)), dim3(SF_THREADS), fixed + (size_t)L.raw_slots * L.raw_bytes + (size_t)L.b_slots * L.b_bytes, st, mapA, mapB, P, L);
    GNN_CHECK_LAUNCH(who);
    return GNN_OK;
}

gnn_status segment_gemm_f32(const char* who, int mode, int slot, const CUtensorMap& mapA, const CUtensorMap& mapB, SegGemmParams& P, cudaStream_t st) {
    return mode == SG_Y ? sf_launch<SG_Y>(who, slot, mapA, mapB, P, st) : mode == SG_DX ? sf_launch<SG_DX>(who, slot, mapA, mapB, P, st) : sf_launch<SG_DW>(who, slot, mapA, mapB, P, st);
}

}  // namespace gnn
