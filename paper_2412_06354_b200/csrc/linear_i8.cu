// Dense transform in 8-bit integers, for answering: rows and output channels carry a scale each,
//   Y[i,m] = act(sx[i] * sw[m] * sum_k xq[i,k] * wq[m,k] + bias[m]),
// and the rounding of rows to 8 bits that makes the operands.  The sums are exact (int32); the products run on the tensor
// cores through the pipeline of segment_gemm.cuh, a few rows on four-product integer instructions.
#include "segment_gemm.cuh"

namespace gnn {

constexpr int I8_SLOT = 54;  // of allow_big_smem: two of them

// ------------------------------------------------------------------ rows to 8 bits
// scale = max |x| / 127, q = x / scale rounded to the nearest integer, ties to even, as the exact quotient would be: the
// estimate, x * (1 / scale) rounded by adding 1.5 * 2^23 (one fma; the integer is in the sum's low bits), is off by less than 1e-4
// of a step, and what remains, r = x - q * scale, is exact in fp32 (a multiple of the last bit of scale, or of half of it where
// q is 1, and at most about half of scale).  Where 2 |r| is under scale, q stands; the few chunks with a value at or beyond the
// half are done again with care.
constexpr float Q_MAGIC = 12582912.f;

struct RowScale {
    float scale, inv, half, start;  // start: where the remainders' maximum begins (above half: all with care)
    uint32_t keep;                  // 0: a row of zeros in the result
    // from the bits of max |x|: not finite -> scale NaN and zeros; scale 0 (or underflown to it) -> zeros
    __device__ __forceinline__ explicit RowScale(uint32_t top) {
        scale = top < 0x7F800000u ? __fdiv_rn(__uint_as_float(top), 127.f) : __uint_as_float(0x7FC00000u);
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(scale));  // 2^-23 of it off: of 127 steps, 2e-5 of a step
        keep = scale > 0.f ? 0xFFFFFFFFu : 0u;
        half = keep ? 0.5f * scale : INFINITY;
        start = tiny() && keep ? INFINITY : 0.f;
    }
    __device__ __forceinline__ bool tiny() const { return scale < 1e-30f; }  // 1 / scale may overflow, scale / 2 may be rounded
    // with care: the neighbour where the remainder passes half a step, the even one where it is half a step
    __device__ __forceinline__ int exact(float x) const {
        float s = scale, i = inv;
        if (tiny()) {  // the same quotient of values 2^80 times as large (exact)
            x *= 1.2089258196146292e24f;
            s *= 1.2089258196146292e24f;
            i = __fdiv_rn(1.f, s);
        }
        float q = fmaf(x, i, Q_MAGIC) - Q_MAGIC;
        const float r = 2.f * fmaf(-q, s, x), a = fabsf(r);
        if (a > s || (a == s && ((int)q & 1))) q += r > 0.f ? 1.f : -1.f;
        return (int)fminf(fmaxf(q, -127.f), 127.f);  // a subnormal scale may be rounded down so far that more steps fit
    }
};

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// largest |x| of a chunk, as bits that order as the values do (what is not finite above all)
template <typename T>
__device__ __forceinline__ uint32_t chunk_top(uint4 v) {
    uint32_t m = 0;
    if constexpr (Chunk<T>::N == 4) {
        m = max(max(v.x & 0x7FFFFFFFu, v.y & 0x7FFFFFFFu), max(v.z & 0x7FFFFFFFu, v.w & 0x7FFFFFFFu));
    } else {  // two bf16 to a word; a NaN wins and becomes 0x7FFF
        auto larger = [](uint32_t a, uint32_t b) {
            uint32_t c;
            asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
            return c;
        };
        const uint32_t a = larger(larger(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), larger(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
        m = max(a << 16, a & 0xFFFF0000u);
    }
    return m;
}
template <typename T>
__device__ __forceinline__ void chunk_out(uint4 v, const RowScale& rs, int8_t* q) {
    constexpr int N = Chunk<T>::N;
    uint32_t w[N / 4];
    float f[N], far = rs.start;
    uint32_t u[N];
    Chunk<T>::unpack(v, f);
    const float2 inv = make_float2(rs.inv, rs.inv), minus = make_float2(-rs.scale, -rs.scale), magic = make_float2(Q_MAGIC, Q_MAGIC);
#pragma unroll
    for (int k = 0; k < N; k += 2) {
        const float2 x = make_float2(f[k], f[k + 1]), e = fma2(x, inv, magic);
        const float2 r = fma2(add2(e, make_float2(-Q_MAGIC, -Q_MAGIC)), minus, x);
        u[k] = __float_as_uint(e.x);
        u[k + 1] = __float_as_uint(e.y);
        far = fmaxf(fmaxf(far, fabsf(r.x)), fabsf(r.y));
    }
    if (far >= rs.half) {  // a value at half a step (of bf16 rows one in 600: half the largest) or one whose estimate fell on the wrong side
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float r = fmaf(-(__uint_as_float(u[k]) - Q_MAGIC), rs.scale, f[k]);
            if (fabsf(r) > rs.half || (fabsf(r) == rs.half && (u[k] & 1u))) u[k] += r > 0.f ? 1 : -1;
        }
        if (rs.start > 0.f) {
#pragma unroll
            for (int k = 0; k < N; ++k) u[k] = (uint32_t)rs.exact(f[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < N / 4; ++k) w[k] = __byte_perm(__byte_perm(u[4 * k], u[4 * k + 1], 0x0040), __byte_perm(u[4 * k + 2], u[4 * k + 3], 0x0040), 0x5410) & rs.keep;
    if constexpr (N == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q) = w[0];
}

// L lanes per row of whole 16-byte chunks, up to CH chunks per lane held in registers between the two passes
template <typename T, int L, int CH>
__global__ void __launch_bounds__(256)
quantize_rows_kernel(const T* X, int64_t N, int K, int8_t* __restrict__ q, float* __restrict__ scale) {
    pdl_wait();
    constexpr int PER = Chunk<T>::N;
    const int64_t row = (blockIdx.x * (int64_t)256 + threadIdx.x) / L;
    const int lane = threadIdx.x % L, chunks = K / PER;
    const bool on = row < N;
    const T* const x = X + row * K;
    uint4 v[CH];
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        v[c] = make_uint4(0, 0, 0, 0);
        if (on && lane + c * L < chunks) v[c] = ld_16(x + (lane + c * L) * PER);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) top = max(top, chunk_top<T>(v[c]));
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if (!on) return;
    const RowScale rs(top);
    if (lane == 0) scale[row] = rs.scale;
#pragma unroll
    for (int c = 0; c < CH; ++c)
        if (lane + c * L < chunks) chunk_out<T>(v[c], rs, q + row * K + (lane + c * L) * PER);
}

// long rows: a block per row, CH chunks per thread in registers
template <typename T, int CH>
__global__ void __launch_bounds__(256)
quantize_long_rows_kernel(const T* X, int64_t N, int K, int8_t* __restrict__ q, float* __restrict__ scale) {
    pdl_wait();
    __shared__ uint32_t tops[2][8];
    constexpr int PER = Chunk<T>::N;
    const int chunks = K / PER;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < N; row += gridDim.x, turn ^= 1) {
        const T* const x = X + row * K;
        uint4 v[CH];
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int i = (int)threadIdx.x + c * 256;
            v[c] = i < chunks ? ld_16(x + i * PER) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) top = max(top, chunk_top<T>(v[c]));
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (threadIdx.x % 32 == 0) tops[turn][threadIdx.x / 32] = top;
        __syncthreads();  // the other half of tops serves the next row: one barrier a row
#pragma unroll
        for (int w = 0; w < 8; ++w) top = max(top, tops[turn][w]);
        const RowScale rs(top);
        if (threadIdx.x == 0) scale[row] = rs.scale;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int i = (int)threadIdx.x + c * 256;
            if (i < chunks) chunk_out<T>(v[c], rs, q + row * K + i * PER);
        }
    }
}

// any K: a block per row, elements one by one, read twice.  170,000 x 100 bf16 160 us (104 features, whole chunks: 11.4 us), 170,000 x 47 fp32 130 us,
// 20,000 x 1001 bf16 50 us: bound by the blocks' latency, eight rows in flight an SM.
template <typename T>
__global__ void __launch_bounds__(256)
quantize_any_kernel(const T* X, int64_t N, int K, int8_t* __restrict__ q, float* __restrict__ scale) {
    pdl_wait();
    __shared__ uint32_t tops[8];
    for (int64_t row = blockIdx.x; row < N; row += gridDim.x) {
        const T* const x = X + row * K;
        uint32_t top = 0;
        for (int k = threadIdx.x; k < K; k += 256) top = max(top, abs_bits((float)x[k]));
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) top = max(top, tops[w]);
        __syncthreads();
        const RowScale rs(top);
        if (threadIdx.x == 0) scale[row] = rs.scale;
        for (int k = threadIdx.x; k < K; k += 256) q[row * K + k] = rs.keep ? (int8_t)rs.exact((float)x[k]) : (int8_t)0;
    }
}

template <typename T>
static void launch_quantize(const T* X, int64_t N, int K, int8_t* q, float* scale, cudaStream_t st) {
    constexpr int PER = Chunk<T>::N;
    const int chunks = K / PER;
    auto run = [&](auto kernel, int lanes) { launch_overlapped(kernel, dim3((unsigned)ceil_div(N * lanes, 256)), dim3(256), 0, st, X, N, K, q, scale); };
    const dim3 rows((unsigned)(N < 148 * 8 ? N : 148 * 8));
    // (a block per row from 512 chunks on: below, 16,384 x 2048 fp32, a block per row takes 41 us)
    if (K % PER == 0 && chunks > 512 && chunks <= 2048) {
        auto run_long = [&](auto kernel) { launch_overlapped(kernel, rows, dim3(256), 0, st, X, N, K, q, scale); };
        chunks <= 1024 ? run_long(quantize_long_rows_kernel<T, 4>) : run_long(quantize_long_rows_kernel<T, 8>);
        return;
    }
    if (K % PER != 0 || chunks > 2048) {
        launch_overlapped(quantize_any_kernel<T>, rows, dim3(256), 0, st, X, N, K, q, scale);
        return;
    }
    // four chunks per lane where the row has them: what a row costs once (the scale, the maximum over its lanes) is shared by 32 values
    // (170,000 x 256 bf16: 23.7 us, 5.5 TB/s; two chunks per lane: 33.7 us)
    if (chunks <= 4) run(quantize_rows_kernel<T, 4, 1>, 4);
    else if (chunks <= 8) run(quantize_rows_kernel<T, 4, 2>, 4);
    else if (chunks <= 16) run(quantize_rows_kernel<T, 4, 4>, 4);
    else if (chunks <= 32) run(quantize_rows_kernel<T, 8, 4>, 8);
    else if (chunks <= 64) run(quantize_rows_kernel<T, 16, 4>, 16);
    else if (chunks <= 128) run(quantize_rows_kernel<T, 32, 4>, 32);
    else if (chunks <= 256) run(quantize_rows_kernel<T, 32, 8>, 32);
    else run(quantize_rows_kernel<T, 32, 16>, 32);
}

// ------------------------------------------------------------------ the product
// A few rows: a warp per output channel and four rows, four products to an instruction.  Bound by reading the weights once: one row,
// 1024 x 1024, 4.3 us, of which about 2.5 are the launch.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256)
linear_i8_rows_kernel(const int8_t* xq, const float* sx, const int8_t* wq, const float* sw, int N, int K, int M, const float* bias, int relu, T* __restrict__ Y, int* status) {
    pdl_wait();
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *status = 0;
    constexpr int R = 4;
    const int lane = threadIdx.x & 31, m = (int)blockIdx.x * 8 + (int)(threadIdx.x >> 5), n0 = (int)blockIdx.y * R;
    if (m >= M) return;
    const int8_t* const w = wq + (int64_t)m * K;
    int acc[R] = {0, 0, 0, 0};
    if constexpr (WIDE) {
#pragma unroll 2
        for (int k = lane * 16; k < K; k += 512) {
            const uint4 a = ld_16(w + k);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (n0 + r >= N) break;
                const uint4 b = ld_16(xq + (int64_t)(n0 + r) * K + k);
                acc[r] = __dp4a((int)a.x, (int)b.x, acc[r]);
                acc[r] = __dp4a((int)a.y, (int)b.y, acc[r]);
                acc[r] = __dp4a((int)a.z, (int)b.z, acc[r]);
                acc[r] = __dp4a((int)a.w, (int)b.w, acc[r]);
            }
        }
    } else {
        for (int k = lane; k < K; k += 32) {
            const int a = w[k];
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (n0 + r < N) acc[r] += a * xq[(int64_t)(n0 + r) * K + k];
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = __reduce_add_sync(0xFFFFFFFFu, acc[r]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (lane != r || n0 + r >= N) continue;
        const float s = sx[n0 + r], b = bias ? bias[m] : 0.f;
        float y = sg_i8_wide(s) ? sg_i8_wide_value(acc[r], s, sw[m], b) : sg_i8_value(acc[r], s, sw[m], b);  // as the tensor-core path rounds
        if (relu) y = y < 0.f ? 0.f : y;
        Y[(int64_t)(n0 + r) * M + m] = T(y);
    }
}

// rows of bytes on 16-byte starts, zeros behind the last (170,000 x 100 -> 47: 26.5 us with it, 112 features without 17.6)
__global__ void __launch_bounds__(256)
pad_bytes_kernel(const int8_t* src, int64_t rows, int cols, int8_t* __restrict__ dst, int ld) {
    pdl_wait();
    const int chunks = ld / 16;
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (i >= rows * chunks) return;
    const int64_t r = i / chunks;
    const int c = (int)(i - r * chunks) * 16;
    union { int8_t b[16]; uint4 v; } u;
#pragma unroll
    for (int k = 0; k < 16; ++k) u.b[k] = c + k < cols ? src[r * cols + c + k] : (int8_t)0;
    *reinterpret_cast<uint4*>(dst + r * ld + c) = u.v;
}

static int up16(int x) { return (x + 15) & ~15; }
// Few rows / the tensor cores: 8 rows of 256 x 256 2.4 / 4.3 us, of 1024 x 1024 3.8 / 6.0, of 2048 x 2048 5.7 / 7.8; 16 rows 2.4 / 4.3, 4.2 / 6.0, 8.9 / 7.8.
static bool i8_few_rows(int32_t N) { return N <= 8; }

struct I8Ws {
    size_t x, w, bytes;
    I8Ws(int64_t N, int K, int M) {
        const bool pads = K % 16 != 0 && !i8_few_rows((int32_t)N);
        x = 256;
        w = x + (pads ? up256((size_t)N * up16(K)) : 0);
        bytes = w + (pads ? up256((size_t)M * up16(K)) : 0);
    }
};

static const int8_t* padded_bytes(const int8_t* src, int64_t rows, int cols, void* dst, cudaStream_t st) {
    const int ld = up16(cols);
    if (ld == cols) return src;
    launch_overlapped(pad_bytes_kernel, dim3((unsigned)ceil_div(rows * (ld / 16), 256)), dim3(256), 0, st, src, rows, cols, (int8_t*)dst, ld);
    return (const int8_t*)dst;
}

}  // namespace gnn

using namespace gnn;

extern "C" {

gnn_status gnn_quantize_rows(const void* X, int32_t N, int K, gnn_dtype dtype, int8_t* q, float* scale, gnn_stream stream) {
    const char* who = "gnn_quantize_rows";
    GNN_REQUIRE(N >= 0 && K > 0, GNN_ERR_INVALID_ARG, "%s: bad shape", who);
    GNN_REQUIRE(dtype == GNN_F32 || dtype == GNN_BF16, GNN_ERR_INVALID_ARG, "%s: bad dtype", who);
    GNN_REQUIRE(K <= INT32_MAX - 256, GNN_ERR_UNSUPPORTED, "%s: K up to 2^31 - 257", who);  // a step of 256 behind the last stays an int
    if (N == 0) return GNN_OK;
    GNN_REQUIRE(X && q && scale, GNN_ERR_INVALID_ARG, "%s: null argument", who);
    GNN_REQUIRE(aligned16(X) && aligned16(q), GNN_ERR_INVALID_ARG, "%s: matrices must be 16-byte aligned", who);
    if (dtype == GNN_F32) launch_quantize((const float*)X, N, K, q, scale, as_stream(stream));
    else launch_quantize((const __nv_bfloat16*)X, N, K, q, scale, as_stream(stream));
    GNN_CHECK_LAUNCH(who);
    return GNN_OK;
}

size_t gnn_linear_i8_workspace(int32_t N, int K, int M) {
    if (N < 0 || K <= 0 || M <= 0) return 0;
    return I8Ws(N, K, M).bytes;
}

gnn_status gnn_linear_i8(const int8_t* xq, const float* x_scale, const int8_t* wq, const float* w_scale, int32_t N, int K, int M, gnn_dtype dtype,
                         const float* bias, int relu, void* Y, void* ws, size_t ws_bytes, gnn_stream stream) {
    const char* who = "gnn_linear_i8";
    GNN_REQUIRE(N >= 0 && K > 0 && M > 0, GNN_ERR_INVALID_ARG, "%s: bad shape", who);
    GNN_REQUIRE(dtype == GNN_F32 || dtype == GNN_BF16, GNN_ERR_INVALID_ARG, "%s: bad dtype", who);
    // 128 * 128 * K stays inside int32
    GNN_REQUIRE(K <= 131071 && N < INT32_MAX - TC_ROWS && M <= INT32_MAX - 256, GNN_ERR_UNSUPPORTED, "%s: K up to 131071, N up to 2^31 - 130, M up to 2^31 - 257", who);
    const I8Ws iw(N, K, M);
    GNN_REQUIRE(ws && ws_bytes >= iw.bytes, GNN_ERR_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes needed", who, iw.bytes);
    cudaStream_t st = as_stream(stream);
    const bool few = i8_few_rows(N);
    if (N == 0) {
        if (cudaMemsetAsync(ws, 0, sizeof(int), st) != cudaSuccess) GNN_FAIL(GNN_ERR_CUDA, "%s: memset failed (is it a device pointer?)", who);
        return GNN_OK;
    }
    GNN_REQUIRE(xq && x_scale && wq && w_scale && Y, GNN_ERR_INVALID_ARG, "%s: null argument", who);
    GNN_REQUIRE(aligned16(xq) && aligned16(wq) && aligned16(Y) && aligned16(ws), GNN_ERR_INVALID_ARG, "%s: matrices and workspace must be 16-byte aligned", who);
    if (few) {
        const dim3 grid((unsigned)ceil_div(M, 8), (unsigned)ceil_div(N, 4));
        auto run = [&](auto kernel, auto* y) { launch_overlapped(kernel, grid, dim3(256), 0, st, xq, x_scale, wq, w_scale, (int)N, K, M, bias, relu, y, (int*)ws); };
        if (dtype == GNN_F32) K % 16 == 0 ? run(linear_i8_rows_kernel<float, true>, (float*)Y) : run(linear_i8_rows_kernel<float, false>, (float*)Y);
        else K % 16 == 0 ? run(linear_i8_rows_kernel<__nv_bfloat16, true>, (__nv_bfloat16*)Y) : run(linear_i8_rows_kernel<__nv_bfloat16, false>, (__nv_bfloat16*)Y);
        GNN_CHECK_LAUNCH(who);
        return GNN_OK;
    }
    GNN_REQUIRE(tensor_map_encoder_available(), GNN_ERR_CUDA, "%s: the driver has no tensor-map encoder", who);
    const int8_t* const xp = padded_bytes(xq, N, K, (char*)ws + iw.x, st);
    const int8_t* const wp = padded_bytes(wq, M, K, (char*)ws + iw.w, st);
    GNN_CHECK_LAUNCH(who);
    SegGemmParams P = {};
    const int64_t row_tiles = ceil_div(N, TC_ROWS);
    P.seg_ptr = nullptr; P.G = 1; P.N = N;
    P.bn = sg_block(M, 256, row_tiles);
    P.tiles_n = (M + P.bn - 1) / P.bn; P.tiles_m = 1;
    P.slices = (K + 127) / 128; P.contraction = K;
    sg_deal(P, (size_t)K * M);
    P.a_rows = N < TC_ROWS ? (N + 7) / 8 * 8 : TC_ROWS;
    P.rows_out = TC_ROWS; P.cols_out = M;
    P.out = Y; P.vec = (size_t)M * elem_size(dtype) % 16 == 0;
    P.bias = bias; P.relu = relu; P.sx = x_scale; P.sw = w_scale;
    P.status = (int*)ws; P.reset = 1;
    CUtensorMap mapA, mapB;
    if (!make_map_planes(&mapA, xp, 1, 1, N, K, up16(K), P.a_rows) || !make_map_planes(&mapB, wp, 1, 1, M, K, up16(K), P.bn))
        GNN_FAIL(GNN_ERR_CUDA, "%s: tensor map encoding failed", who);
    return dtype == GNN_F32 ? sg_launch<SG_I8, float>(who, I8_SLOT, mapA, mapB, P, 0, st) : sg_launch<SG_I8, __nv_bfloat16>(who, I8_SLOT + 1, mapA, mapB, P, 0, st);
}

}  // extern "C"
