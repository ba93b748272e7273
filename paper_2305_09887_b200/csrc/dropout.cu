// Dropout whose mask is never stored: an element is kept or dropped by 16 bits of a hash of (seed, row id, column), so the
// backward pass, another kernel or another cut of the graph into parts finds the same mask again.
//     h = S(S(seed) ^ (id << 32 | column / 4)),  S = one SplitMix64 step;  lane = 16 bits number column % 4 of h
//     y = residual + (lane >= t ? x / (1 - t / 65536) : 0),  t = round(65536 p)
#include "rows.cuh"

namespace {

struct DropoutArgs {
    const void* X;
    const void* residual;
    void* Y;
    int64_t n, ldx, ldr, ldy;
    int d, units;       // columns; groups of eight columns in a row
    int vx, vr, vy;     // granules of the rows (bytes)
    DropArgs drop;
};

// Bound by memory: a thread brings eight values by one load and hashes twice for them, rows and units go round the whole grid so that
// neighbouring threads have neighbouring units.  5M x 128 in bf16 with ids and a residual: 660 us, 5.85 TB/s.
template <class T>
__global__ void __launch_bounds__(256) dropout_kernel(const DropoutArgs a) {
    wait_for_kernel_before();
    const T* X = static_cast<const T*>(a.X);
    const T* R = static_cast<const T*>(a.residual);
    T* Y = static_cast<T*>(a.Y);
    const int64_t stride = (int64_t)gridDim.x * blockDim.x, at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t step_rows = stride / a.units;
    const int step_units = (int)(stride - step_rows * a.units);
    int64_t r = at / a.units;
    int u = (int)(at - r * a.units);
    while (r < a.n) {
        const int valid = min(8, a.d - 8 * u);
        Eight<T> x;
        x.load(X + r * a.ldx + 8 * u, valid, a.vx);
        float v[8];
        x.values(v);
        if (a.drop.threshold) drop_eight(a.drop, a.drop.ids ? (uint32_t)__ldg(a.drop.ids + r) : (uint32_t)r, u, v);
        if (R) {
            Eight<T> y;
            y.load(R + r * a.ldr + 8 * u, valid, a.vr);
            float w[8];
            y.values(w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += w[j];
        }
        store_eight(Y + r * a.ldy + 8 * u, v, valid, a.vy);
        r += step_rows;
        u += step_units;
        if (u >= a.units) {
            u -= a.units;
            ++r;
        }
    }
}

}  // namespace

extern "C" int32_t rtma_dropout(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t d, const void* X, int64_t ldx, const int32_t* row_ids,
                                const void* residual, int64_t ldr, double p, uint64_t seed, void* Y, int64_t ldy, void* stream_) {
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    if (dtype < RTMA_F32 || dtype > RTMA_F16) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_dropout: dtype=%d", dtype);
    if (n < 0 || n >= (int64_t(1) << 31) || d < 0) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_dropout: n=%lld d=%d", (long long)n, d);
    if (!(p >= 0.0 && p <= 1.0)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_dropout: p=%g outside [0,1]", p);
    if (n == 0 || d == 0) return RTMA_OK;
    if (!X || !Y) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_dropout: null pointer");
    if (ldx < d || ldy < d || (residual && ldr < d)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_dropout: rows of %d values lie closer than that", d);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    RTMA_TRY(prepare_row_call(ctx, 0, stream));
    const size_t es = row_type_bytes(dtype);
    DropoutArgs a{X, residual, Y, n, ldx, ldr, ldy, d, (int)ceil_div(d, 8), row_granule(X, ldx, es), row_granule(residual, ldr, es),
                  row_granule(Y, ldy, es), drop_args(p, seed, row_ids)};
    const int64_t blocks = ceil_div(n * a.units, 256);
    const unsigned grid = (unsigned)(blocks < (int64_t)ctx->sm_count * 32 ? blocks : (int64_t)ctx->sm_count * 32);
    auto kernel = dtype == RTMA_F32 ? dropout_kernel<float> : dtype == RTMA_BF16 ? dropout_kernel<__nv_bfloat16> : dropout_kernel<__half>;
    {
        KernelScope ks(ctx, KC_POST, stream);
        launch_kernel(kernel, grid, 256, 0, stream, a);
    }
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}
