// Layers over the rows of many parts (layer.cu) of fp32 rows: the kernel of grouped_split.cu with the layer behind its sums.
//
// The two matrices of a gated layer are laid out by turns of 32 columns when they are split into planes: the 64 columns of a tile that a
// warp drains are then 32 results, and a lane has both factors of each of its own.
#include <algorithm>

#include "grouped_split.cuh"
#include "layer.cuh"

RTMA_BOUNDS_TU()

namespace {

using namespace grouped;
using namespace grouped::split;

// fp32 matrices [d_in][halves * width] -> planes [part][3][d_in][ld]; halves == 2: by turns of 32 columns, ld a multiple of 64
__global__ void __launch_bounds__(256) layer_planes_kernel(const float* __restrict__ W, int64_t w_stride, int parts, int d_in, int width, int halves, int granule, int ld,
                                                           __nv_bfloat16* __restrict__ planes) {
    wait_for_kernel_before();
    const int units = ld / 8;
    const int64_t matrix = (int64_t)ld * d_in, total = (int64_t)parts * d_in * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / units;
        const int u = (int)(i - row * units);
        const int64_t part = row / d_in, r = row - part * d_in;
        const int second = halves == 2 ? u >> 2 & 1 : 0, c = halves == 2 ? 32 * (u >> 3) + 8 * (u & 3) : 8 * u;
        Eight<float> x;
        x.load(W + part * w_stride + (r * halves + second) * width + (c < width ? c : 0), max(0, min(8, width - c)), granule);
        uint4 p[3];
        split_eight(reinterpret_cast<const uint32_t(&)[8]>(x.w), p);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(planes + (3 * part + k) * matrix + r * ld + 8 * u) = p[k];
    }
}

template <int EASY, bool GATED, bool GRADIENT>
__global__ void __launch_bounds__(THREADS, BLOCKS_PER_SM) layer_split_kernel(const __grid_constant__ LayerArgs a) {
    typedef Form<FORWARD> F;
    __shared__ SplitShared<FORWARD> sh;
    LayerBias bias{sh.bias + 64 * (threadIdx.x >> 5)};
    split_body<FORWARD, EASY>(a, sh, [&](const Walk<FORWARD, BM, BK>& out, float (&total)[F::HALVES][32], int group, int out_m, int out_c, int lane) {
        static_assert(F::HALVES == 2, "64 columns a warp");
        const int rows = min(32, out.rows - out_m);
        const int64_t row0 = out.row0 + out_m;
        // the columns of total[h]: results, or (gated) what they are made of
        auto column = [&](int h) { return GATED ? (out.n0 + out_c) / 2 : out.n0 + out_c + 32 * h; };
        auto columns = [&](int h) { return GATED ? min(32, a.width - column(0)) : min(min(32, a.BN - out_c - 32 * h), a.width - column(h)); };
        bias.fetch(a, out.part, out.n0, 2, lane, static_cast<const float*>(nullptr), [&](int h) { return column(h) + (GATED && h ? a.width : 0); }, columns);
        const float slope = a.slope ? __ldg(a.slope + out.part * a.slope_stride) : 0.f;
        float slope_sum = 0.f;
#pragma unroll
        for (int h = 0; h < (GATED ? 1 : 2); ++h) {
            const int c = column(h), cols = columns(h);
            if (rows <= 0 || cols <= 0) continue;
            const float* const from = static_cast<const float*>(a.side) + (row0 + lane) * a.lds + c;
            float ds = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f2 z[4], y[4], d[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    z[k] = pack2(total[h][8 * q + 2 * k], total[h][8 * q + 2 * k + 1]);
                    if constexpr (GATED) y[k] = pack2(total[1][8 * q + 2 * k], total[1][8 * q + 2 * k + 1]);
                }
                if (GRADIENT || a.side) {
                    Eight<float> e;
                    e.load(from + 8 * q, lane < rows ? max(0, min(8, cols - 8 * q)) : 0, a.gs);
                    pairs_of(e, d);
                }
                ds += eight_results<GATED, GRADIENT>(a.act, a.side != nullptr, bias, (GATED ? 0 : 32 * h) + 8 * q, 32 + 8 * q, slope, a.slope_slots != nullptr, cols - 8 * q, z, y, d);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    unpack2(z[k], total[h][8 * q + 2 * k], total[h][8 * q + 2 * k + 1]);
                    if constexpr (GATED && GRADIENT) unpack2(y[k], total[1][8 * q + 2 * k], total[1][8 * q + 2 * k + 1]);
                }
            }
            if (lane < rows) slope_sum += ds;
            float* const to = static_cast<float*>(a.out) + row0 * a.ldo + c;
            put_rows(to, a.ldo, a.go, total[h], rows, cols, lane);
            if constexpr (GATED && GRADIENT) put_rows(to + a.width, a.ldo, a.g2, total[1], rows, cols, lane);
        }
        if (GRADIENT && a.slope_slots) {
            for (int o = 16; o > 0; o >>= 1) slope_sum += __shfl_xor_sync(0xffffffffu, slope_sum, o);
            if (lane == 0) a.slope_slots[(int64_t)out.tile * a.slope_warps + 4 * group + (threadIdx.x >> 5 & 3)] = slope_sum;
        }
    });
}

template <int EASY, bool GATED, bool GRADIENT>
int32_t launch_form(rtma_ctx* ctx, const LayerArgs& a, unsigned grid, bool& configured, cudaStream_t stream) {
    void (*kernel)(LayerArgs) = layer_split_kernel<EASY, GATED, GRADIENT>;
    if (!configured) {
        RTMA_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Form<FORWARD>::DYNAMIC_BYTES));
        configured = true;
    }
    launch_kernel(kernel, grid, THREADS, Form<FORWARD>::DYNAMIC_BYTES, stream, a);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

int plane_columns(const LayerArgs& a, bool gated) { return gated ? (int)ceil_div(a.width, 32) * 64 : (int)ceil_div(a.width, 8) * 8; }

}  // namespace

size_t layer_split_bytes(const LayerArgs& a, bool gated) { return (size_t)3 * 2 * (a.w_stride ? a.G : 1) * a.d_in * plane_columns(a, gated); }

void describe_layer_split(LayerArgs& a, bool gated) {
    a.va = row_granule(a.A, a.lda, 4);
    a.vb = std::min(row_granule(a.B, a.ldb, 4), row_granule(nullptr, a.w_stride, 4));
    a.g2 = std::min(a.go, row_granule(nullptr, a.width, 4));
    a.tile_rows = BM;
    a.tiles = a.n / BM + a.G;
    const int N = gated ? plane_columns(a, true) : a.width;
    a.n_tiles = (int)ceil_div(N, SPLIT_COLUMNS);
    a.BN = gated ? std::min(N, SPLIT_COLUMNS) : (int)ceil_div(ceil_div(N, a.n_tiles), 16) * 16;
    a.n_tiles = (int)ceil_div(N, a.BN);
    a.slope_warps = a.BN > Form<FORWARD>::COLUMNS ? 8 : 4;
}

int32_t launch_layer_split(rtma_ctx* ctx, LayerArgs& a, bool gated, bool gradient, void* planes, int cls, cudaStream_t stream) {
    const int64_t tiles = a.tiles * a.n_tiles;
    if (tiles >= (int64_t(1) << 30)) return rtma_fail(ctx, RTMA_ERR_OVERFLOW, "grouped layer: %lld tiles", (long long)tiles);
    const int parts = a.w_stride ? a.G : 1, ld = plane_columns(a, gated), halves = gated ? 2 : 1;
    if (!make_tensor_map_16bit(&a.map_b, true, planes, 3 * (uint64_t)parts, a.d_in, ld, ld, (uint64_t)ld * a.d_in, BK, 64, 3))
        return rtma_fail(ctx, RTMA_ERR_CUDA, "grouped layer: no tensor map for %d matrices of %d x %d", parts, a.d_in, a.width);
    {
        const int64_t blocks = ceil_div((int64_t)parts * a.d_in * (ld / 8), 256);
        KernelScope ks(ctx, KC_WEIGHT_PREP, stream);
        launch_kernel(layer_planes_kernel, (unsigned)std::min<int64_t>(blocks, 16 * ctx->sm_count), 256, 0, stream, static_cast<const float*>(a.B), a.w_stride, parts, a.d_in,
                      a.width, halves, std::min(a.vb, halves == 2 ? row_granule(nullptr, a.width, 4) : 32), ld, static_cast<__nv_bfloat16*>(planes));
        RTMA_LAUNCH_CHECK(ctx);
    }
    const unsigned grid = (unsigned)std::min<int64_t>(tiles, (int64_t)BLOCKS_PER_SM * ctx->sm_count);
    bool* once = ctx->layer_configured + 24;
    KernelScope ks(ctx, cls, stream);
    auto launch = [&](auto EASY) {
        constexpr int easy = decltype(EASY)::value;
        bool* at = once + 4 * easy;
        if (gated) return gradient ? launch_form<easy, true, true>(ctx, a, grid, at[3], stream) : launch_form<easy, true, false>(ctx, a, grid, at[2], stream);
        return gradient ? launch_form<easy, false, true>(ctx, a, grid, at[1], stream) : launch_form<easy, false, false>(ctx, a, grid, at[0], stream);
    };
    // rows on 16-byte boundaries with widths of whole 16 bytes are loaded without a case for every value
    return a.va >= 16 && a.d_in % 4 == 0 ? launch(std::integral_constant<int, 1>()) : launch(std::integral_constant<int, 0>());
}
