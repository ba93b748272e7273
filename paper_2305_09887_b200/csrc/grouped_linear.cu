// The product of every part's rows with the part's own matrix, and its gradients:
//   forward  Y[r] = X[r] W_g + b_g        dx  dX[r] = dY[r] W_g^T        dw  dW_g = sum_r X[r]^T dY[r], db_g = sum_r dY[r]
// for the rows r of part g.  Simple form: 64 x 64 tiles on the fp32 units.
#include "rows.cuh"

RTMA_BOUNDS_TU()

namespace {

constexpr int BM = 64, BN = 64, BK = 16, THREADS = 256;

struct LinearArgs {
    const int64_t* offsets;
    int64_t n;
    int G, span;
    int64_t tile_rows, tiles;
    int d_in, d_out;
    const void *A, *B;  // rows; matrices (forward, dx) or rows (dw)
    int64_t lda, ldb, w_stride;
    const void* bias;
    int64_t bias_stride;
    void* out;
    int64_t ldo;
    float* partial;  // dw: [tile][(d_in + 1) * d_out], the last row the bias's
    float *dW, *db;
    int64_t dw_stride, db_stride;
};

template <class T, bool TRANSPOSED>
__global__ void __launch_bounds__(THREADS) linear_rows_kernel(const LinearArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    __shared__ float sa[BK][BM + 1], sb[BK][BN + 1];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums, a.span);
    const int tile = blockIdx.x;
    if (tile >= tile_start[a.G]) return;
    const int part = part_of_tile(tile_start, a.G, tile);
    int64_t begin, end;
    part_rows(a.offsets, a.n, part, begin, end);
    begin += (int64_t)(tile - tile_start[part]) * a.tile_rows;
    const int rows = (int)min(end - begin, a.tile_rows);
    const int K = TRANSPOSED ? a.d_out : a.d_in, N = TRANSPOSED ? a.d_in : a.d_out, n0 = blockIdx.y * BN;
    const T* A = static_cast<const T*>(a.A) + begin * a.lda;
    const T* W = static_cast<const T*>(a.B) + part * a.w_stride;
    const T* bias = a.bias ? static_cast<const T*>(a.bias) + part * a.bias_stride : nullptr;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += BK) {
        for (int i = threadIdx.x; i < BM * BK; i += THREADS) {
            const int k = i % BK, m = i / BK;
            sa[k][m] = m < rows && k0 + k < K ? to_f32(A[m * a.lda + k0 + k]) : 0.f;
        }
        for (int i = threadIdx.x; i < BN * BK; i += THREADS) {
            const int j = TRANSPOSED ? i / BK : i % BN, k = TRANSPOSED ? i % BK : i / BN;
            const bool ok = k0 + k < K && n0 + j < N;
            sb[k][j] = ok ? to_f32(TRANSPOSED ? W[(int64_t)(n0 + j) * a.d_out + k0 + k] : W[(int64_t)(k0 + k) * a.d_out + n0 + j]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < BK; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
    T* out = static_cast<T*>(a.out) + begin * a.ldo;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = ty + 16 * i, c = n0 + tx + 16 * j;
            if (m < rows && c < N) out[m * a.ldo + c] = from_f32<T>(acc[i][j] + (bias ? to_f32(bias[c]) : 0.f));
        }
}

template <class T>
__global__ void __launch_bounds__(THREADS) linear_weights_kernel(const LinearArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    __shared__ float sa[BK][BM + 1], sb[BK][BN + 1];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums, a.span);
    const int tile = blockIdx.x;
    if (tile >= tile_start[a.G]) return;
    const int part = part_of_tile(tile_start, a.G, tile);
    int64_t begin, end;
    part_rows(a.offsets, a.n, part, begin, end, a.span);
    begin += (int64_t)(tile - tile_start[part]) * a.tile_rows;
    end = min(end, begin + a.tile_rows);
    const int m0 = blockIdx.z * BM, n0 = blockIdx.y * BN;
    const T* X = static_cast<const T*>(a.A);
    const T* dY = static_cast<const T*>(a.B);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {}, sums[4] = {};
    for (int64_t r0 = begin; r0 < end; r0 += BK) {
        for (int i = threadIdx.x; i < BM * BK; i += THREADS) {
            const int m = i % BM, k = i / BM;
            sa[k][m] = r0 + k < end && m0 + m < a.d_in ? to_f32(X[(r0 + k) * a.lda + m0 + m]) : 0.f;
        }
        for (int i = threadIdx.x; i < BN * BK; i += THREADS) {
            const int j = i % BN, k = i / BN;
            sb[k][j] = r0 + k < end && n0 + j < a.d_out ? to_f32(dY[(r0 + k) * a.ldb + n0 + j]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < BK; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sums[j] += sb[k][tx + 16 * j];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][j] = fmaf(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
            }
        __syncthreads();
    }
    float* out = a.partial + (int64_t)tile * (a.d_in + 1) * a.d_out;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = n0 + tx + 16 * j;
        if (c >= a.d_out) continue;
        if (ty == 0 && m0 == 0) out[(int64_t)a.d_in * a.d_out + c] = sums[j];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (m0 + ty + 16 * i < a.d_in) out[(int64_t)(m0 + ty + 16 * i) * a.d_out + c] = acc[i][j];
    }
}

// The tiles' sums of every part added up in order.
__global__ void __launch_bounds__(THREADS) linear_reduce_kernel(const LinearArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums, a.span);
    const int part = blockIdx.y;
    const int64_t weights = (int64_t)a.d_in * a.d_out, count = weights + a.d_out, i = (int64_t)blockIdx.x * THREADS + threadIdx.x;
    if (i >= count) return;
    float s = 0.f;
    for (int t = tile_start[part]; t < tile_start[part + 1]; ++t) s += a.partial[(int64_t)t * count + i];
    if (i < weights) a.dW[part * a.dw_stride + i] = s;
    else if (a.db) a.db[part * a.db_stride + i - weights] = s;
}

template <class K>
K by_type(int32_t dtype, K f32, K bf16, K f16) { return dtype == RTMA_F32 ? f32 : dtype == RTMA_BF16 ? bf16 : f16; }

int32_t check_linear(rtma_ctx* ctx, const char* who, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out) {
    RTMA_TRY(check_parts(ctx, who, n, G, offsets));
    if (dtype < RTMA_F32 || dtype > RTMA_F16) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: dtype=%d", who, dtype);
    if (d_in < 1 || d_out < 1 || d_in > RTMA_MAX_WIDTH || d_out > RTMA_MAX_WIDTH)
        return rtma_fail(ctx, RTMA_ERR_UNSUPPORTED, "%s: %d x %d outside [1,%d]", who, d_in, d_out, RTMA_MAX_WIDTH);
    return RTMA_OK;
}

int32_t run_rows(rtma_ctx* ctx, const char* who, bool transposed, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                 const void* A, int64_t lda, const void* W, int64_t w_stride, const void* b, int64_t b_stride, void* out, int64_t ldo, void* stream_) {
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_linear(ctx, who, dtype, n, G, offsets, d_in, d_out));
    if (n == 0) return RTMA_OK;
    if (!A || !W || !out) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: null pointer", who);
    const int K = transposed ? d_out : d_in, N = transposed ? d_in : d_out;
    if (lda < K || ldo < N) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: rows of %d and %d values lie closer than that", who, K, N);
    if (A == out) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: the result must not overlap the rows", who);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    RTMA_TRY(prepare_row_call(ctx, 0, stream));
    LinearArgs a{};
    a.offsets = offsets; a.n = n; a.G = G; a.span = 1;
    a.tile_rows = BM;
    a.tiles = n / BM + G;
    a.d_in = d_in; a.d_out = d_out;
    a.A = A; a.lda = lda; a.B = W; a.w_stride = w_stride; a.bias = b; a.bias_stride = b_stride;
    a.out = out; a.ldo = ldo;
    auto kernel = transposed ? by_type(dtype, &linear_rows_kernel<float, true>, &linear_rows_kernel<__nv_bfloat16, true>, &linear_rows_kernel<__half, true>)
                             : by_type(dtype, &linear_rows_kernel<float, false>, &linear_rows_kernel<__nv_bfloat16, false>, &linear_rows_kernel<__half, false>);
    {
        KernelScope ks(ctx, transposed ? KC_GEMM_DGRAD : KC_GEMM_FWD, stream);
        launch_kernel(kernel, dim3((unsigned)a.tiles, (unsigned)ceil_div(N, BN)), THREADS, 0, stream, a);
    }
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

}  // namespace

extern "C" int32_t rtma_grouped_linear(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                                       const void* X, int64_t ldx, const void* W, int64_t w_stride, const void* b, int64_t b_stride, void* Y,
                                       int64_t ldy, void* stream) {
    return run_rows(ctx, "rtma_grouped_linear", false, dtype, n, G, offsets, d_in, d_out, X, ldx, W, w_stride, b, b_stride, Y, ldy, stream);
}

extern "C" int32_t rtma_grouped_linear_dx(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                                          const void* dY, int64_t lddy, const void* W, int64_t w_stride, void* dX, int64_t lddx, void* stream) {
    return run_rows(ctx, "rtma_grouped_linear_dx", true, dtype, n, G, offsets, d_in, d_out, dY, lddy, W, w_stride, nullptr, 0, dX, lddx, stream);
}

extern "C" int32_t rtma_grouped_linear_dw(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                                          const void* X, int64_t ldx, const void* dY, int64_t lddy, float* dW, int64_t dw_stride, float* db,
                                          int64_t db_stride, void* stream_) {
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_linear(ctx, "rtma_grouped_linear_dw", dtype, n, G, offsets, d_in, d_out));
    if (!dW || (n > 0 && (!X || !dY))) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_grouped_linear_dw: null pointer");
    if (ldx < d_in || lddy < d_out) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_grouped_linear_dw: rows of %d and %d values lie closer than that", d_in, d_out);
    const int64_t weights = (int64_t)d_in * d_out;
    const bool shared = G > 1 && dw_stride == 0;
    if (G > 1 && db && (db_stride == 0) != shared)
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_grouped_linear_dw: either both gradients are one for all parts or neither");
    if (G > 1 && !shared && ((dw_stride < weights && dw_stride > -weights) || (db && db_stride < d_out && db_stride > -d_out)))
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_grouped_linear_dw: gradients of the parts overlap");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    LinearArgs a{};
    a.offsets = offsets; a.n = n;
    a.G = shared ? 1 : G;
    a.span = shared ? G : 1;
    const int64_t blocks = ceil_div(d_in, BM) * ceil_div(d_out, BN), chunk = ceil_div(n * blocks, 8 * (int64_t)ctx->sm_count);
    a.tile_rows = chunk < 256 ? 256 : ceil_div(chunk, 64) * 64;
    a.tiles = n / a.tile_rows + a.G;
    a.d_in = d_in; a.d_out = d_out;
    a.A = X; a.lda = ldx; a.B = dY; a.ldb = lddy;
    a.dW = dW; a.dw_stride = dw_stride; a.db = db; a.db_stride = db_stride;
    RTMA_TRY(prepare_row_call(ctx, sizeof(float) * a.tiles * (weights + d_out), stream));
    a.partial = reinterpret_cast<float*>(ctx->arena);
    if (n > 0) {
        auto kernel = by_type(dtype, &linear_weights_kernel<float>, &linear_weights_kernel<__nv_bfloat16>, &linear_weights_kernel<__half>);
        KernelScope ks(ctx, KC_GEMM_WGRAD, stream);
        launch_kernel(kernel, dim3((unsigned)a.tiles, (unsigned)ceil_div(d_out, BN), (unsigned)ceil_div(d_in, BM)), THREADS, 0, stream, a);
    }
    RTMA_LAUNCH_CHECK(ctx);
    {
        KernelScope ks(ctx, KC_REDUCE_SGD, stream);
        launch_kernel(linear_reduce_kernel, dim3((unsigned)ceil_div(weights + d_out, THREADS), (unsigned)a.G), THREADS, 0, stream, a);
    }
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}
