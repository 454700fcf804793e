// Dense transform whose weight depends on the row's segment (the node types or relations of a heterogeneous graph):
//   Y[i,:] = act(X[i,:] * W[g(i)] + bias[g(i)]),  dX[i,:] = dY[i,:] * W[g(i)]^T,  dW[g] = X_g^T * dY_g
// Entry points, their workspaces and the small kernels around the products of segment_gemm.cuh: padded copies of matrices
// whose rows do not start on 16 bytes, the three bf16 terms of fp32 weights, the ordered sum of dW's partials.
#include "segment_gemm.cuh"

namespace gnn {

constexpr int LS_SLOT = 48;  // of allow_big_smem: six of them

// Rows of fp32 as three planes of bf16 rows (x = x1 + x2 + x3 exactly): a thread writes 8 elements of each plane.  Rows of dst
// are ld elements apart; what follows the last column is zero.
__global__ void __launch_bounds__(256)
split_rows_kernel(const float* src, int64_t rows, int cols, __nv_bfloat16* __restrict__ dst, int ld, int vec) {
    pdl_wait();
    const int chunks = ld / 8;
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (i >= rows * chunks) return;
    const int64_t r = i / chunks;
    const int c = (int)(i - r * chunks) * 8;
    float x[8];
    const float* const p = src + r * cols + c;
    if (vec && c + 8 <= cols) {
        Chunk<float>::unpack(ld_16(p), x);
        Chunk<float>::unpack(ld_16(p + 4), x + 4);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = c + k < cols ? p[k] : 0.f;
    }
#pragma unroll
    for (int l = 0; l < 3; ++l) {
        const uint4 v = Chunk<__nv_bfloat16>::pack(x);
        *reinterpret_cast<uint4*>(dst + (l * rows + r) * (int64_t)ld + c) = v;
        float t[8];
        Chunk<__nv_bfloat16>::unpack(v, t);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] -= t[k];  // exact: the rounded term shares the leading bits
    }
}

// rows on 16-byte starts, zeros behind the last column: a chunk of PER elements per thread
template <typename E, int PER>
__global__ void __launch_bounds__(256)
widen_rows_kernel(const E* src, int64_t rows, int cols, E* __restrict__ dst, int chunks) {
    pdl_wait();
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (i >= rows * chunks) return;
    const int64_t r = i / chunks;
    const int c = (int)(i - r * chunks) * PER;
    union { E e[PER]; uint4 v; } u;
#pragma unroll
    for (int k = 0; k < PER; ++k) u.e[k] = c + k < cols ? src[r * cols + c + k] : E(0);
    *reinterpret_cast<uint4*>(dst + (r * chunks) * PER + c) = u.v;
}

// dW of the segments that more than one part holds (their partials in a fixed order: R runs of consecutive parts, each in
// ascending order with eight loads in flight, then the runs in ascending order) or none (zeros).  A block of 256 threads:
// 256 / R of them side by side with V elements each.  Eight runs where segments have many parts, few elements each (one run: 25 us
// of the 62 us of the fp32 gradients of 40,000 x 128 x 64, eight: 4 us); one run otherwise (bf16 gradients of 100,000 x 256 x 256,
// seven parts a segment: eight runs 3 us slower).
template <typename T, int V, int R>
__global__ void __launch_bounds__(256)
segment_sum_kernel(const int64_t* seg_ptr, int G, int64_t N, int64_t part_rows, const float* part, int64_t size, T* __restrict__ dW) {
    pdl_wait();
    constexpr int E = 256 / R * V;
    __shared__ float runs[R > 1 ? R : 1][R > 1 ? E : 1];
    const int lane = threadIdx.x % (256 / R), run = threadIdx.x / (256 / R);
    for (int g = blockIdx.y; g < G; g += gridDim.y) {
        int64_t a = seg_ptr[g], b = seg_ptr[g + 1];
        a = a < 0 ? 0 : a > N ? N : a;
        b = b < 0 ? 0 : b > N ? N : b;
        const int64_t first = a / part_rows, last = (b - 1) / part_rows;
        if (b > a && first == last) continue;  // written by the product
        const int64_t e0 = blockIdx.x * (int64_t)E, e = e0 + lane * V;
        float s[V];
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] = 0.f;
        if (b > a && e < size) {
            const int64_t per = (last - first + R) / R, p0 = first + run * per, p1 = p0 + per <= last ? p0 + per : last + 1;
            for (int64_t p = p0; p < p1; p += 8) {
                float v[8][V];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    // the first part holds the segment's start (cut at the part's end: odd), the others begin inside it (even)
                    const int64_t q = p + u, at = (2 * q + (q == first && a >= first * part_rows ? 1 : 0)) * size + e;
                    if constexpr (V == 4) {
                        const float4 w = q < p1 ? *reinterpret_cast<const float4*>(part + at) : make_float4(0.f, 0.f, 0.f, 0.f);
                        v[u][0] = w.x; v[u][1] = w.y; v[u][2] = w.z; v[u][3] = w.w;
                    } else {
                        v[u][0] = q < p1 ? part[at] : 0.f;
                    }
                }
#pragma unroll
                for (int u = 0; u < 8; ++u)
#pragma unroll
                    for (int k = 0; k < V; ++k) s[k] += v[u][k];
            }
        }
        if constexpr (R == 1) {
            if (e < size) {
                T* const to = dW + g * size + e;
#pragma unroll
                for (int k = 0; k < V; ++k) to[k] = T(s[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) runs[run][lane * V + k] = s[k];
            __syncthreads();
            for (int k = threadIdx.x; k < E; k += 256)
                if (e0 + k < size) {
                    float t = runs[0][k];
#pragma unroll
                    for (int q = 1; q < R; ++q) t += runs[q][k];
                    dW[g * size + e0 + k] = T(t);
                }
            __syncthreads();
        }
    }
}

static int up8(int x) { return (x + 7) & ~7; }
// elements between rows that start on 16 bytes
static int apart(int cols, gnn_dtype dtype) { return dtype == GNN_F32 ? (cols + 3) & ~3 : up8(cols); }

// How the rows are cut for dW: parts x tiles blocks of work on 148 SMs.  Few parts mean few partials; as many as keep the SMs
// busy: the smallest number whose last wave costs at most 5 % over the best of all numbers, parts of at least 256 rows.  And of
// at most 2048 rows in fp32, as the forward product's contraction: every 16 rows the accumulator cuts off what lies under the last bit of a
// 24-bit sum, measured up to 0.9 * 2^-24 of the result (terms of one sign made for it: 1.35e-5 over 4096 rows, 6.8e-6 over 2048; others half of
// that).  bf16: 65536 rows, 2^-12, under the rounding.
static int64_t dw_parts(int64_t N, int64_t tiles, bool f32) {
    const int64_t longest = f32 ? 2048 : 65536, least = N > longest ? ceil_div(N, longest) : 1;
    int64_t most = N / 256;
    if (most > 296) most = 296;
    if (most < least) most = least;
    auto cost = [&](int64_t p) { return (double)ceil_div(p * tiles, 148) / (double)p; };
    double best = cost(least);
    for (int64_t p = least + 1; p <= most; ++p) best = cost(p) < best ? cost(p) : best;
    for (int64_t p = least; p <= most; ++p)
        if (cost(p) <= 1.05 * best) return p;
    return least;
}

struct SegWs {
    size_t x, dy, w, part, bytes;
    int64_t parts;
    int bn, tiles_n, tiles_m;
    SegWs(int64_t N, int G, int K, int M, gnn_dtype dtype, bool forward) {
        const bool f32 = dtype == GNN_F32;
        auto copy = [&](int64_t rows, int cols) -> size_t { return apart(cols, dtype) != cols ? up256((size_t)elem_size(dtype) * rows * apart(cols, dtype)) : 0; };
        x = 256;
        dy = x + copy(N, K);
        w = dy + (forward ? 0 : copy(N, M));
        part = w + (f32 ? up256((size_t)6 * G * K * up8(M)) : copy((int64_t)G * K, M));
        bytes = part;
        bn = sg_block(M, f32 ? 128 : 256, 148);
        tiles_n = (M + bn - 1) / bn;
        tiles_m = (K + 127) / 128;
        parts = dw_parts(N, (int64_t)tiles_n * tiles_m, f32);
        if (!forward && parts > 1) bytes += (size_t)2 * parts * K * M * 4;
    }
};

// the matrix with rows on 16 bytes: itself or its copy at dst
static const void* operand(const void* src, int64_t rows, int cols, gnn_dtype dtype, void* dst, cudaStream_t st) {
    const int ld = apart(cols, dtype);
    if (cols == ld) return src;
    const int chunks = ld * elem_size(dtype) / 16;
    const dim3 grid((unsigned)ceil_div(rows * chunks, 256));
    if (dtype == GNN_F32) launch_overlapped(widen_rows_kernel<float, 4>, grid, dim3(256), 0, st, (const float*)src, rows, cols, (float*)dst, chunks);
    else launch_overlapped(widen_rows_kernel<uint16_t, 8>, grid, dim3(256), 0, st, (const uint16_t*)src, rows, cols, (uint16_t*)dst, chunks);
    return dst;
}
// the weights: bf16 as above, fp32 as three planes
static const void* weights(const void* W, int64_t rows, int M, gnn_dtype dtype, void* dst, cudaStream_t st) {
    if (dtype == GNN_BF16) return operand(W, rows, M, dtype, dst, st);
    launch_overlapped(split_rows_kernel, dim3((unsigned)ceil_div(rows * (up8(M) / 8), 256)), dim3(256), 0, st, (const float*)W, rows, M, (__nv_bfloat16*)dst, up8(M), (int)(M % 4 == 0));
    return dst;
}

static const char* seg_shape_error(int32_t N, int G, int K, int M, gnn_dtype dtype) {
    if (N < 0 || G < 0 || K <= 0 || M <= 0) return "bad shape";
    if (dtype != GNN_F32 && dtype != GNN_BF16) return "bad dtype";
    return nullptr;
}
static bool seg_size_ok(int32_t N, int G, int K, int M, gnn_dtype dtype) {
    const int most = dtype == GNN_F32 ? 2048 : 8192;
    return K <= most && M <= most && N < INT32_MAX - TC_ROWS && (int64_t)G * K <= ((int64_t)1 << 31) - 1 && G <= (1 << 24);
}

// Y = X * W (dx = false) or dX = dY * W^T (dx = true): in [N, cin], out [N, cout]
static gnn_status seg_rows(const char* who, bool dx, const void* in, const void* w, const int64_t* seg_ptr, int32_t N, int G, int K, int M, gnn_dtype dtype,
                           const float* bias, int relu, void* out, int* status, int reset, cudaStream_t st) {
    const bool f32 = dtype == GNN_F32;
    const int cin = dx ? M : K, cout = dx ? K : M;
    SegGemmParams P = {};
    const int64_t row_tiles = (int64_t)N / TC_ROWS + G;
    P.seg_ptr = seg_ptr; P.G = G; P.N = N;
    P.bn = sg_block(cout, f32 ? 128 : 256, row_tiles);
    P.tiles_n = (cout + P.bn - 1) / P.bn; P.tiles_m = 1;
    P.slices = (cin + 63) / 64; P.contraction = cin;
    sg_deal(P, (size_t)G * K * M * (f32 ? 6 : 2), !f32);
    P.a_rows = N < TC_ROWS ? (N + 7) / 8 * 8 : TC_ROWS;
    P.rows_out = TC_ROWS; P.cols_out = cout;
    P.out = out; P.vec = (size_t)cout * elem_size(dtype) % 16 == 0;
    P.bias = bias; P.relu = relu; P.status = status; P.reset = reset;
    CUtensorMap mapA, mapB;
    if (!make_map_planes(&mapA, in, f32 ? 2 : 0, 1, N, cin, apart(cin, dtype), P.a_rows) ||
        !make_map_planes(&mapB, w, 0, (int64_t)(f32 ? 3 : 1) * G, K, M, up8(M), dx ? P.bn : 64))
        GNN_FAIL(GNN_ERR_CUDA, "%s: tensor map encoding failed", who);
    if (f32) return segment_gemm_f32(who, dx ? SG_DX : SG_Y, LS_SLOT + dx, mapA, mapB, P, 0, st);
    return dx ? sg_launch<SG_DX, __nv_bfloat16>(who, LS_SLOT + 2, mapA, mapB, P, 0, st) : sg_launch<SG_Y, __nv_bfloat16>(who, LS_SLOT + 3, mapA, mapB, P, 0, st);
}

static gnn_status zero(const char* who, void* p, size_t bytes, cudaStream_t st) {
    if (bytes && cudaMemsetAsync(p, 0, bytes, st) != cudaSuccess) GNN_FAIL(GNN_ERR_CUDA, "%s: memset failed (is it a device pointer?)", who);
    return GNN_OK;
}

}  // namespace gnn

using namespace gnn;

extern "C" {

size_t gnn_linear_segments_workspace(int32_t N, int G, int K, int M, gnn_dtype dtype, int backward) {
    if (seg_shape_error(N, G, K, M, dtype)) return 0;
    return SegWs(N, G, K, M, dtype, !backward).bytes;
}

gnn_status gnn_linear_segments(const void* X, const int64_t* seg_ptr, const void* W, int32_t N, int G, int K, int M, gnn_dtype dtype,
                               const float* bias, int relu, void* Y, void* ws, size_t ws_bytes, gnn_stream stream) {
    const char* who = "gnn_linear_segments";
    const char* bad = seg_shape_error(N, G, K, M, dtype);
    GNN_REQUIRE(!bad, GNN_ERR_INVALID_ARG, "%s: %s", who, bad);
    GNN_REQUIRE(seg_size_ok(N, G, K, M, dtype), GNN_ERR_UNSUPPORTED, "%s: K and M up to 8192 (fp32: 2048), G K under 2^31", who);
    GNN_REQUIRE(ws && ws_bytes >= 256, GNN_ERR_WORKSPACE_TOO_SMALL, "%s: workspace too small", who);
    cudaStream_t st = as_stream(stream);
    const gnn_status rs = zero(who, ws, N == 0 || G == 0 ? sizeof(int) : 0, st);
    if (rs != GNN_OK || N == 0) return rs;
    GNN_REQUIRE(Y, GNN_ERR_INVALID_ARG, "%s: null Y", who);
    if (G == 0) return zero(who, Y, (size_t)N * M * elem_size(dtype), st);
    GNN_REQUIRE(X && W && seg_ptr, GNN_ERR_INVALID_ARG, "%s: null argument", who);
    GNN_REQUIRE(aligned16(X) && aligned16(W) && aligned16(Y) && aligned16(ws), GNN_ERR_INVALID_ARG, "%s: matrices and workspace must be 16-byte aligned", who);
    const SegWs sw(N, G, K, M, dtype, true);
    GNN_REQUIRE(ws_bytes >= sw.bytes, GNN_ERR_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes needed", who, sw.bytes);
    GNN_REQUIRE(tensor_map_encoder_available(), GNN_ERR_CUDA, "%s: the driver has no tensor-map encoder", who);
    char* const w8 = (char*)ws;
    const void* Xp = operand(X, N, K, dtype, w8 + sw.x, st);
    const void* Wp = weights(W, (int64_t)G * K, M, dtype, w8 + sw.w, st);
    GNN_CHECK_LAUNCH(who);
    return seg_rows(who, false, Xp, Wp, seg_ptr, N, G, K, M, dtype, bias, relu, Y, (int*)ws, 1, st);
}

gnn_status gnn_linear_segments_backward(const void* X, const int64_t* seg_ptr, const void* W, const void* dY, int32_t N, int G, int K, int M,
                                        gnn_dtype dtype, void* dX, void* dW, void* ws, size_t ws_bytes, gnn_stream stream) {
    const char* who = "gnn_linear_segments_backward";
    const char* bad = seg_shape_error(N, G, K, M, dtype);
    GNN_REQUIRE(!bad, GNN_ERR_INVALID_ARG, "%s: %s", who, bad);
    GNN_REQUIRE(seg_size_ok(N, G, K, M, dtype), GNN_ERR_UNSUPPORTED, "%s: K and M up to 8192 (fp32: 2048), G K under 2^31", who);
    const SegWs sw(N, G, K, M, dtype, false);
    GNN_REQUIRE(ws && ws_bytes >= sw.bytes, GNN_ERR_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes needed", who, sw.bytes);
    cudaStream_t st = as_stream(stream);
    const size_t s = (size_t)elem_size(dtype);
    if (N == 0 || G == 0) {
        gnn_status rc = zero(who, ws, sizeof(int), st);
        if (rc == GNN_OK && dX) rc = zero(who, dX, (size_t)N * K * s, st);
        if (rc == GNN_OK && dW) rc = zero(who, dW, (size_t)G * K * M * s, st);
        return rc;
    }
    GNN_REQUIRE(dY && seg_ptr, GNN_ERR_INVALID_ARG, "%s: null argument", who);
    GNN_REQUIRE(!dX || W, GNN_ERR_INVALID_ARG, "%s: dX needs W", who);
    GNN_REQUIRE(!dW || X, GNN_ERR_INVALID_ARG, "%s: dW needs X", who);
    GNN_REQUIRE(aligned16(dY) && (!dX || (aligned16(W) && aligned16(dX))) && (!dW || (aligned16(X) && aligned16(dW))) && aligned16(ws), GNN_ERR_INVALID_ARG,
                "%s: matrices and workspace must be 16-byte aligned", who);
    GNN_REQUIRE(tensor_map_encoder_available(), GNN_ERR_CUDA, "%s: the driver has no tensor-map encoder", who);
    if (!dX && !dW) return zero(who, ws, sizeof(int), st);
    char* const w8 = (char*)ws;
    const bool f32 = dtype == GNN_F32;
    const void* dYp = operand(dY, N, M, dtype, w8 + sw.dy, st);
    int reset = 1;
    if (dX) {
        const void* Wp = weights(W, (int64_t)G * K, M, dtype, w8 + sw.w, st);
        GNN_CHECK_LAUNCH(who);
        const gnn_status rc = seg_rows(who, true, dYp, Wp, seg_ptr, N, G, K, M, dtype, nullptr, 0, dX, (int*)ws, reset, st);
        if (rc != GNN_OK) return rc;
        reset = 0;
    }
    if (dW) {
        const void* Xp = operand(X, N, K, dtype, w8 + sw.x, st);
        GNN_CHECK_LAUNCH(who);
        SegGemmParams P = {};
        P.seg_ptr = seg_ptr; P.G = G; P.N = N;
        P.bn = sw.bn; P.tiles_n = sw.tiles_n; P.tiles_m = sw.tiles_m;
        P.part_rows = ceil_div(N, sw.parts);
        P.units = ceil_div(N, P.part_rows) * P.tiles_n * P.tiles_m;
        P.rows_out = K; P.cols_out = M;
        P.out = dW; P.vec = (size_t)M * s % 16 == 0;
        P.part = (float*)(w8 + sw.part);
        P.status = (int*)ws; P.reset = reset;
        CUtensorMap mapA, mapB;
        const int type = f32 ? 2 : 0, box_rows = f32 ? 32 : 64;
        if (!make_map_planes(&mapA, Xp, type, 1, N, K, apart(K, dtype), box_rows) || !make_map_planes(&mapB, dYp, type, 1, N, M, apart(M, dtype), box_rows))
            GNN_FAIL(GNN_ERR_CUDA, "%s: tensor map encoding failed", who);
        const int64_t part_rows_all = sw.parts > 1 ? 2 * sw.parts * K : 1;  // (one part: no partials)
        const gnn_status rc = f32 ? segment_gemm_f32(who, SG_DW, LS_SLOT + 4, mapA, mapB, P, part_rows_all, st)
                                  : sg_launch<SG_DW, __nv_bfloat16>(who, LS_SLOT + 5, mapA, mapB, P, part_rows_all, st);
        if (rc != GNN_OK) return rc;
        const int64_t size = (int64_t)K * M;
        auto sum = [&](auto kernel, auto* to, int elements) {
            launch_overlapped(kernel, dim3((unsigned)ceil_div(size, (int64_t)elements), (unsigned)(G < 65535 ? G : 65535)), dim3(256), 0, st, seg_ptr, G, (int64_t)N, P.part_rows,
                              (const float*)P.part, size, to);
        };
        const bool four = size % 4 == 0, many = sw.parts >= 16 * (int64_t)G;
        auto pick = [&](auto* to) {
            using T = typename std::remove_pointer<decltype(to)>::type;
            if (many) four ? sum(segment_sum_kernel<T, 4, 8>, to, 128) : sum(segment_sum_kernel<T, 1, 8>, to, 32);
            else four ? sum(segment_sum_kernel<T, 4, 1>, to, 1024) : sum(segment_sum_kernel<T, 1, 1>, to, 256);
        };
        if (f32) pick((float*)dW); else pick((__nv_bfloat16*)dW);
        GNN_CHECK_LAUNCH(who);
    }
    return GNN_OK;
}

}  // extern "C"
