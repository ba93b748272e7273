// Layers over the rows of many parts, on the tensor cores:
//   Y[r] = R[r] + act(X[r] W_g + b_g)                          gated: H[r] = R[r] + act(X[r] V_g + c_g) * (X[r] U_g + d_g)
// for the rows r of part g, W_g = [V_g | U_g] in a gated layer, and the first step of their gradients,
//   dZ[r] = dY[r] act'(Z[r])                                   gated: dZ[r] = [dH u act'(v) | dH act(v)]
// with Z = X W + b worked out again from the inputs: kept from the forward pass it would cost a write there and a read here, which is
// more than the product as long as the contraction has fewer terms than about 600 (16-bit rows).  dX = dZ W^T and dW = X^T dZ are then the
// grouped products of grouped_linear.cu.
//
// One kernel body (grouped_rows.cuh) for all four: the product stays in tensor memory and goes through the layer in the registers of
// the warps that drain it.  A tile of a gated layer has the same columns of both matrices, so that a lane finds both factors of a result in its own
// row.  dZ is rounded to the rows' type: it is an operand of 16-bit products.
//
// This file: the calls.  The kernels of 16-bit rows are in layer_kernels.cuh, those of fp32 rows in layer_split.cu.
#include <algorithm>

#include "layer.cuh"

RTMA_BOUNDS_TU()

namespace {

using namespace grouped;

constexpr int BM = 128, BK = 64;  // of the kernels on 16-bit rows

// 16-bit matrices -> [part][d_in][halves * up] on 16-byte boundaries, up: width rounded up to 8
__global__ void __launch_bounds__(256) lay_out_matrices_kernel(const __half* __restrict__ W, int64_t w_stride, int parts, int d_in, int width, int halves, int granule,
                                                               __half* __restrict__ out) {
    wait_for_kernel_before();
    const int units = (width + 7) / 8;
    const int64_t total = (int64_t)parts * d_in * halves * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t run = i / units, row = run / halves, part = row / d_in;  // run: a row of one matrix
        const int u = (int)(i - run * units), h = (int)(run - row * halves);
        Eight<__half> x;
        x.load(W + part * w_stride + ((row - part * d_in) * halves + h) * width + 8 * u, min(8, width - 8 * u), granule);
        *reinterpret_cast<uint4*>(out + 8 * i) = x.w[0];
    }
}

struct SumsArgs {
    const int64_t* offsets;
    int64_t n, tile_rows, tiles;
    int G, places, n_tiles, columns;  // columns: 0 if their sums are not wanted
    int width, real_width;            // of one of dZ's halves, with and without what was rounded up
    const float *column_slots, *slope_slots;
    void* db;
    float* dslope;
    int64_t db_stride, dslope_stride;
    bool shared, slope_shared;
    // a column's place in the bias, or -1
    __device__ __forceinline__ int place_of(int column) const {
        const int second = column >= width ? 1 : 0, c = column - second * width;
        return c < real_width ? second * real_width + c : -1;
    }
};

// What pairs of blocks leave of sums over rows (layer_pairs.cuh), added up in order: a block for 32 columns of dZ and a part (or all parts:
// shared), the last of a part for its slope's gradient.
template <class O>
__global__ void __launch_bounds__(256) layer_sums_kernel(const __grid_constant__ SumsArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    __shared__ double red[256];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool of_slope = (int)blockIdx.x * 32 >= a.columns, shared = of_slope ? a.slope_shared : a.shared;
    if ((int)blockIdx.y > 0 && shared) return;
    const int column = 32 * blockIdx.x + lane, first = shared ? 0 : blockIdx.y, last = shared ? a.G : first + 1;
    const int64_t tiles = tile_start[a.G];
    double s = 0.0;
    for (int part = first; part < last; ++part) {
        const int from = tile_start[part], to = tile_start[part + 1];
        if (from == to) continue;
        // the places whose tiles [tiles i / places, tiles (i + 1) / places) are among the part's
        int i = (int)((int64_t)from * a.places / tiles);
        while ((int)(tiles * (i + 1) / a.places) <= from) ++i;
        for (; i < a.places && (int)(tiles * i / a.places) < to; ++i) {
            if ((int)(tiles * i / a.places) == (int)(tiles * (i + 1) / a.places)) continue;
            const int64_t slot = 8 * (int64_t)(i + part);
            if (!of_slope) s += column < a.columns ? a.column_slots[(slot + warp) * a.columns + column] : 0.f;
            else
                for (int k = threadIdx.x; k < 32 * a.n_tiles; k += 256) s += a.slope_slots[slot * 4 * a.n_tiles + k];
        }
    }
    red[threadIdx.x] = s;
    __syncthreads();
    if (!of_slope) {
        if (warp) return;
        for (int k = 1; k < 8; ++k) s += red[32 * k + lane];
        if (column < a.columns && a.place_of(column) >= 0) static_cast<O*>(a.db)[blockIdx.y * a.db_stride + a.place_of(column)] = from_f32<O>((float)s);
    } else if (threadIdx.x == 0) {
        for (int k = 1; k < 256; ++k) s += red[k];
        a.dslope[blockIdx.y * a.dslope_stride] = (float)s;
    }
}

// What the warps of all tiles have of the slopes' gradients, added up in order; one block for every part, or one for all (shared).
__global__ void __launch_bounds__(256) slope_reduce_kernel(const int64_t* offsets, int64_t n, int G, int64_t tile_rows, int64_t tiles, int64_t per_tile,
                                                           const float* __restrict__ slots, bool shared, float* dslope, int64_t stride) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    __shared__ double red[8];
    wait_for_kernel_before();
    number_tiles(offsets, n, G, tile_rows, tiles, tile_start, warp_sums);
    const int part = blockIdx.x;
    const int64_t from = shared ? 0 : tile_start[part] * per_tile, to = tile_start[shared ? G : part + 1] * per_tile;
    double s = 0.0;
#pragma unroll 4
    for (int64_t i = from + threadIdx.x; i < to; i += 256) s += slots[i];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < 8; ++k) s += red[k];
        dslope[part * stride] = (float)s;
    }
}

// The layer's kernel on 16-bit rows.  room: scratch for the laid-out matrices.
int32_t launch_layer(rtma_ctx* ctx, LayerArgs& a, bool bf16, bool gated, bool gradient, char* room, int cls, cudaStream_t stream) {
    const int halves = gated ? 2 : 1;
    if (room) {
        const int parts = a.w_stride ? a.G : 1;
        const int64_t blocks = ceil_div((int64_t)parts * a.d_in * halves * ceil_div(a.width, 8), 256);
        KernelScope ks(ctx, KC_WEIGHT_PREP, stream);
        launch_kernel(lay_out_matrices_kernel, (unsigned)std::min<int64_t>(blocks, 16 * ctx->sm_count), 256, 0, stream, static_cast<const __half*>(a.B), a.w_stride, parts,
                      a.d_in, a.width, halves, std::min(a.vb, row_granule(nullptr, a.width, 2)), reinterpret_cast<__half*>(room));
        RTMA_LAUNCH_CHECK(ctx);
        a.B = room;
        a.up = (int)ceil_div(a.width, 8) * 8;
        a.ldb = halves * a.up;
        a.w_stride = a.w_stride ? a.d_in * a.ldb : 0;
        a.vb = 16;
    }
    const int64_t tiles = a.tiles * a.n_tiles;
    if (tiles >= (int64_t(1) << 30)) return rtma_fail(ctx, RTMA_ERR_OVERFLOW, "grouped layer: %lld tiles", (long long)tiles);
    a.in_bulk = 2;
    if (!make_tensor_map_16bit(&a.map_b, bf16, a.B, a.w_stride ? a.G : 1, a.d_in, gated ? a.up + a.width : a.width, a.ldb, a.w_stride ? a.w_stride : a.d_in * a.ldb, BK))
        return rtma_fail(ctx, RTMA_ERR_CUDA, "grouped layer: no tensor map for %d matrices of %d x %d", a.w_stride ? a.G : 1, a.d_in, a.width);
    if (a.va >= 16) {
        if (make_tensor_map_16bit(&a.map_a, bf16, a.A, 1, a.n, a.d_in, a.lda, a.n * a.lda, BM)) a.in_bulk |= 1;
        else if (a.places) return rtma_fail(ctx, RTMA_ERR_CUDA, "grouped layer: no tensor map for rows of %d values", a.d_in);
    }
    if (a.places && a.side && !make_store_map(&a.map_side, bf16 ? RTMA_BF16 : RTMA_F16, a.side, a.n, a.width, a.lds))
        return rtma_fail(ctx, RTMA_ERR_CUDA, "grouped layer: no tensor map for rows of %d values", a.width);
    KernelScope ks(ctx, cls, stream);
    const unsigned grid = a.places ? 2u * a.places * a.n_tiles : (unsigned)std::min<int64_t>(tiles, ctx->sm_count);
    return (bf16 ? launch_layer_bf16 : launch_layer_f16)(ctx, a, a.places != 0, gated, gradient, grid, stream);
}

int32_t check_layer(rtma_ctx* ctx, const char* who, const rtma_layer_desc* d, int64_t n, int32_t G, const int64_t* offsets, const float* slope) {
    if (!d) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: null description", who);
    RTMA_TRY(check_parts(ctx, who, n, G, offsets));
    if (d->dtype < RTMA_F32 || d->dtype > RTMA_F16) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: dtype=%d", who, d->dtype);
    if (d->act < RTMA_ACT_NONE || d->act > RTMA_ACT_SILU) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: act=%d", who, d->act);
    if (d->act == RTMA_ACT_PRELU && !slope) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: PReLU without a slope", who);
    const int64_t wide = d->gated ? 2 * (int64_t)d->d_out : d->d_out;
    if (d->d_in < 1 || d->d_out < 1 || d->d_in > RTMA_MAX_WIDTH || wide > RTMA_MAX_WIDTH)
        return rtma_fail(ctx, RTMA_ERR_UNSUPPORTED, "%s: %d x %lld outside [1,%d]", who, d->d_in, (long long)wide, RTMA_MAX_WIDTH);
    return RTMA_OK;
}

// The arguments of the layer's kernel and the scratch that it takes (lay: the matrices have to be laid out).
void describe(rtma_ctx* ctx, LayerArgs& a, const rtma_layer_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx, const void* W, const void* b,
              const float* slope, const void* side, int64_t lds, size_t* bytes) {
    const size_t es = row_type_bytes(d->dtype);
    const int wide = d->gated ? 2 * d->d_out : d->d_out;
    a.error_word = ctx->error_word;
    a.offsets = offsets; a.n = n; a.G = G; a.span = 1;
    a.tile_rows = BM;
    a.tiles = n / BM + G;
    a.m_tiles = 1;
    a.d_in = d->d_in; a.d_out = a.width = a.up = d->d_out;
    a.A = X; a.lda = ldx; a.B = W; a.ldb = wide; a.w_stride = d->w_stride;
    a.bias = b; a.bias_stride = d->b_stride;
    a.va = row_granule(X, ldx, es);
    a.vb = std::min(row_granule(W, wide, es), row_granule(nullptr, d->w_stride, es));
    a.act = d->act;
    a.slope = d->act == RTMA_ACT_PRELU ? slope : nullptr; a.slope_stride = d->slope_stride;
    a.slope_warps = 8;
    a.side = side; a.lds = lds; a.gs = side ? row_granule(side, lds, es) : 0;
    if (d->dtype == RTMA_F32) {
        describe_layer_split(a, d->gated != 0);
        *bytes = layer_split_bytes(a, d->gated != 0);
        return;
    }
    a.bias_up = a.bias_width = a.width;
    // Rows on 16-byte boundaries: pairs of blocks, as long as there are pairs for all tiles of columns
    const int widest = d->gated ? 128 : 256, pairs = ctx->sm_count / 2;
    a.n_tiles = (int)ceil_div(a.width, widest);
    if (a.va >= 16 && (!side || a.gs >= 16) && a.n_tiles <= pairs) {
        a.half = (int)ceil_div(ceil_div(a.width, a.n_tiles), d->gated ? 16 : 32) * 16;
        a.n_tiles = (int)ceil_div(a.width, d->gated ? a.half : 2 * a.half);
        a.tile_rows = 2 * BM;
        a.tiles = n / a.tile_rows + G;
        a.places = (int)std::min<int64_t>(pairs / a.n_tiles, a.tiles);
    } else {
        a.BN = (int)ceil_div(ceil_div(a.width, a.n_tiles), 16) * 16;
        a.n_tiles = (int)ceil_div(a.width, a.BN);
    }
    const bool lay = a.vb < 16 || a.w_stride < 0 || (d->gated && a.width % 8);
    *bytes = lay ? (size_t)2 * (a.w_stride ? G : 1) * a.d_in * (d->gated ? 2 : 1) * ceil_div(a.width, 8) * 8 : 0;
}

}  // namespace

extern "C" int32_t rtma_grouped_layer(rtma_ctx* ctx, const rtma_layer_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx, const void* W,
                                      const void* b, const float* slope, const void* residual, int64_t ldr, void* Y, int64_t ldy, void* stream_) {
    const char* who = "rtma_grouped_layer";
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_layer(ctx, who, d, n, G, offsets, slope));
    if (n == 0) return RTMA_OK;
    if (!X || !W || !Y) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: null pointer", who);
    if (ldx < d->d_in || ldy < d->d_out || (residual && ldr < d->d_out))
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: rows of %d and %d values lie closer than that", who, d->d_in, d->d_out);
    if (X == Y) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: the result must not overlap the rows", who);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    const size_t es = row_type_bytes(d->dtype);
    LayerArgs a{};
    size_t bytes = 0;
    describe(ctx, a, d, n, G, offsets, X, ldx, W, b, slope, residual, ldr, &bytes);
    a.out = Y; a.ldo = ldy;
    a.go = row_granule(Y, ldy, es);
    a.vo = d->dtype != RTMA_F32 && a.go >= 16 && make_store_map(&a.map_o, d->dtype, Y, n, d->d_out, ldy);
    RTMA_TRY(prepare_row_call(ctx, bytes, stream));
    if (d->dtype == RTMA_F32) return launch_layer_split(ctx, a, d->gated != 0, false, ctx->arena, KC_GEMM_FWD, stream);
    return launch_layer(ctx, a, d->dtype == RTMA_BF16, d->gated != 0, false, bytes ? ctx->arena : nullptr, KC_GEMM_FWD, stream);
}

extern "C" int32_t rtma_grouped_layer_grad(rtma_ctx* ctx, const rtma_layer_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx, const void* W,
                                           const void* b, const float* slope, const void* dY, int64_t lddy, void* dZ, int64_t lddz, void* dX, int64_t lddx, void* dW,
                                           int64_t dw_stride, void* db, int64_t db_stride, float* dslope, int64_t dslope_stride, void* stream_) {
    const char* who = "rtma_grouped_layer_grad";
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_layer(ctx, who, d, n, G, offsets, slope));
    const bool gated = d->gated != 0, plain = !gated && d->act == RTMA_ACT_NONE;  // plain: dZ is dY
    const int wide = gated ? 2 * d->d_out : d->d_out;
    if (n > 0 && (!X || !W || !dY || (!plain && !dZ))) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: null pointer", who);
    if (db && !dW) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: the bias gradient comes with the weights'", who);
    if (G > 1 && db && (db_stride == 0) != (dw_stride == 0))
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: either both gradients are one for all parts or neither", who);
    if (G > 1 && db && db_stride != 0 && db_stride < wide && db_stride > -wide) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: gradients of the parts overlap", who);
    if (dslope && d->act != RTMA_ACT_PRELU) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: a slope's gradient without PReLU", who);
    if (d->grad_dtype != d->dtype && d->grad_dtype != RTMA_F32) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: gradients of the parameters in type %d", who, d->grad_dtype);
    if (ldx < d->d_in || lddy < d->d_out || (!plain && lddz < wide) || (dX && lddx < d->d_in))
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: rows of %d and %d values lie closer than that", who, d->d_in, wide);
    if (!plain && n > 0 && (dZ == X || (dZ == dY && (gated || lddz != lddy)) || dZ == dX))
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: dZ must not overlap other rows", who);
    if (n > 0 && dX && (dX == X || (dX == dY && plain))) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: dX must not overlap rows that are still read", who);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    const size_t es = row_type_bytes(d->dtype);
    const void* dz = plain ? dY : dZ;
    const int64_t ldz = plain ? lddy : lddz;
    LayerArgs a{};
    size_t matrices = 0, slots = 0, rows_bytes = 0, dw_bytes = 0;
    describe(ctx, a, d, n, G, offsets, X, ldx, W, b, slope, dY, lddy, &matrices);
    matrices = ArenaCursor::granule(matrices);
    const bool pairs = !plain && n > 0 && a.places != 0, sums = pairs && db;  // the bias gradient comes with dZ
    size_t column_bytes = 0;
    if (pairs) {
        a.columns = wide;
        const size_t rows = 8 * (size_t)(a.places + G);
        column_bytes = sums ? ArenaCursor::granule(rows * wide * sizeof(float)) : 0;
        slots = column_bytes + (dslope ? rows * a.n_tiles * 4 * sizeof(float) : 0);
    } else if (dslope) {
        slots = sizeof(float) * (size_t)(a.tiles * a.n_tiles) * a.slope_warps;
    }
    // all scratch at once: inside a capture nothing is enqueued unless everything fits
    if (dX) RTMA_TRY(grouped_rows(ctx, who, true, d->dtype, n, G, offsets, d->d_in, wide, dz, ldz, W, d->w_stride, nullptr, 0, dX, lddx, &rows_bytes, stream));
    const bool by_pairs = d->dtype != RTMA_F32 && row_granule(X, ldx, es) >= 16 && row_granule(dz, ldz, es) >= 16;
    auto weights = by_pairs ? layer_dw : grouped_dw;
    if (dW)
        RTMA_TRY(weights(ctx, who, d->dtype, n, G, offsets, d->d_in, wide, X, ldx, dz, ldz, d->grad_dtype, dW, dw_stride, sums ? nullptr : db, db_stride, &dw_bytes, stream));
    RTMA_TRY(prepare_row_call(ctx, std::max(plain ? 0 : matrices + slots, std::max(rows_bytes, dw_bytes)), stream));
    if (!plain && n > 0) {
        a.out = dZ; a.ldo = lddz;
        a.go = row_granule(dZ, lddz, es);
        a.g2 = std::min(a.go, row_granule(nullptr, d->d_out, es));
        a.vo = d->dtype != RTMA_F32 && a.go >= 16 && make_store_map(&a.map_o, d->dtype, dZ, n, wide, lddz);
        a.column_slots = sums ? reinterpret_cast<float*>(ctx->arena + matrices) : nullptr;
        a.slope_slots = dslope ? reinterpret_cast<float*>(ctx->arena + matrices + column_bytes) : nullptr;
        if (d->dtype == RTMA_F32) RTMA_TRY(launch_layer_split(ctx, a, gated, true, ctx->arena, KC_GEMM_FWD, stream));
        else RTMA_TRY(launch_layer(ctx, a, d->dtype == RTMA_BF16, gated, true, matrices ? ctx->arena : nullptr, KC_GEMM_FWD, stream));
    }
    const bool slope_shared = G > 1 && dslope_stride == 0;
    if (pairs && (sums || dslope)) {
        SumsArgs m{};
        m.offsets = offsets; m.n = n; m.tile_rows = a.tile_rows; m.tiles = a.tiles;
        m.G = G; m.places = a.places; m.n_tiles = a.n_tiles; m.columns = sums ? wide : 0;
        m.width = a.width; m.real_width = d->d_out;
        m.column_slots = a.column_slots; m.slope_slots = a.slope_slots;
        m.db = db; m.dslope = dslope; m.db_stride = db_stride; m.dslope_stride = dslope_stride;
        m.shared = G > 1 && db_stride == 0; m.slope_shared = slope_shared;
        void (*kernel)(SumsArgs) = d->grad_dtype == RTMA_F32 ? layer_sums_kernel<float> : d->grad_dtype == RTMA_BF16 ? layer_sums_kernel<__nv_bfloat16> : layer_sums_kernel<__half>;
        KernelScope ks(ctx, KC_REDUCE_SGD, stream);
        launch_kernel(kernel, dim3((unsigned)(ceil_div(m.columns, 32) + (dslope ? 1 : 0)), (unsigned)G), 256, 0, stream, m);
        RTMA_LAUNCH_CHECK(ctx);
    } else if (dslope) {
        const int64_t per_tile = (int64_t)a.n_tiles * a.slope_warps;
        KernelScope ks(ctx, KC_REDUCE_SGD, stream);
        launch_kernel(slope_reduce_kernel, slope_shared ? 1u : (unsigned)G, 256, 0, stream, offsets, n, G, a.tile_rows, a.tiles, per_tile,
                      const_cast<const float*>(a.slope_slots), slope_shared, dslope, dslope_stride);
        RTMA_LAUNCH_CHECK(ctx);
    }
    if (dX) RTMA_TRY(grouped_rows(ctx, who, true, d->dtype, n, G, offsets, d->d_in, wide, dz, ldz, W, d->w_stride, nullptr, 0, dX, lddx, nullptr, stream));
    if (dW) RTMA_TRY(weights(ctx, who, d->dtype, n, G, offsets, d->d_in, wide, X, ldx, dz, ldz, d->grad_dtype, dW, dw_stride, sums ? nullptr : db, db_stride, nullptr, stream));
    return RTMA_OK;
}
