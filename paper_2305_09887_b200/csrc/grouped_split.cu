// Grouped products (grouped_linear.cu) of fp32 rows on the tensor cores.
//
// A value is split into three bf16 numbers (8 + 8 + 8 bits, the whole significand) and a product is six MMAs; the three left out are
// below 2^-22 of it.  The tensor cores truncate when they accumulate: a stage of 32 terms starts a fresh accumulator, the five small
// products first, and is then added up in registers, rounded to nearest.
//
// The matrices are split beforehand, once a call, into planes in the scratch, and come by bulk-tensor loads in forward and dx; in dw
// both operands are rows.  The rows' values are split by the warps, which do everything in turn: split the next stage's values
// (which wait in registers) into shared memory, request the ones after, take their columns of the stage before from tensor memory
// and add them up.  When those are there, that stage's place in the ring and its accumulator are free again; warp 0 issues the MMAs,
// warp 1 the loads of W.  All these steps are short and wait for one another, so two blocks share an SM, each on tiles of 128 x 128
// (dw: 128 x 64): one block of twice the width on the SM, which splits less, took 127 us for 200,000 x 128 -> 256 and 220 for the
// 256 x 47 gradient of as many rows (two: 103).
//
// Bound by the chain of these steps, not by the six MMAs (47 us) or the bytes (48) of the first: 200,000 x 128 -> 256 125 us, its dx 133, the
// gradient of 256 x 256 295 (90 TFLOP/s of fp32 products).  Of the first, shared memory's data path is busy for 62 % of the cycles, the
// tensor pipes for 29 %, memory for 24 %, and instructions are issued in 35 %; of the 256 x 47 gradient 46, 15, 34 and 46 %.  The dx kernels
// spill 16 bytes a thread, the others nothing.
#include "grouped_split.cuh"

RTMA_BOUNDS_TU()

namespace {

using namespace grouped;
using namespace grouped::split;

// fp32 matrices -> planes [part][3][d_in][ld] (ld: d_out rounded up to 8)
__global__ void __launch_bounds__(256) split_planes_kernel(const float* __restrict__ W, int64_t w_stride, int parts, int d_in, int d_out, int granule,
                                                           __nv_bfloat16* __restrict__ planes) {
    wait_for_kernel_before();
    const int units = (d_out + 7) / 8;
    const int64_t ld = 8 * (int64_t)units, matrix = ld * d_in, total = (int64_t)parts * d_in * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / units;
        const int u = (int)(i - row * units);
        const int64_t part = row / d_in, r = row - part * d_in;
        Eight<float> x;
        x.load(W + part * w_stride + r * d_out + 8 * u, min(8, d_out - 8 * u), granule);
        uint4 p[3];
        split_eight(reinterpret_cast<const uint32_t(&)[8]>(x.w), p);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(planes + (3 * part + k) * matrix + r * ld + 8 * u) = p[k];
    }
}

template <int MODE, int EASY>
__global__ void __launch_bounds__(THREADS, BLOCKS_PER_SM) split_kernel(const __grid_constant__ LinearArgs a) {
    typedef Form<MODE> F;
    constexpr bool DW = MODE == WEIGHT_GRADIENT;
    __shared__ SplitShared<MODE> sh;
    BiasHolder<float> bias{sh.bias + 64 * (threadIdx.x >> 5)};
    split_body<MODE, EASY>(a, sh, [&](const Walk<MODE, BM, BK>& out, float (&total)[F::HALVES][32], int group, int out_m, int out_c, int lane) {
        const int N = MODE == INPUT_GRADIENT ? a.d_in : MODE == FORWARD ? a.d_out : (int)a.ldo;  // (dw: the slots' rows are padded)
        const int rows = min(32, (DW ? min(BM, a.d_in - out.m0) : out.rows) - out_m);
        const int64_t row0 = (DW ? (int64_t)out.row_tile * (a.d_in + a.bias_rows) + out.m0 : out.row0) + out_m;
        if (MODE == FORWARD && a.bias) bias.fetch(a, out.part, out.n0, F::HALVES * group, 1, min(F::HALVES * (group + 1), (a.BN + 31) / 32), lane);
#pragma unroll
        for (int h = 0; h < F::HALVES; ++h) {
            const int c = out.n0 + out_c + 32 * h, cols = min(min(32, a.BN - out_c - 32 * h), N - c);
            if (rows > 0 && cols > 0) {
                if (MODE == FORWARD && a.bias) bias.add(total[h], h);
                put_rows(static_cast<float*>(a.out) + row0 * a.ldo + c, a.ldo, a.go, total[h], rows, cols, lane);
            }
        }
    });
}

template <int MODE, int EASY>
int32_t launch_form(rtma_ctx* ctx, const LinearArgs& a, unsigned grid, bool& configured, cudaStream_t stream) {
    if (!configured) {
        RTMA_CUDA(ctx, cudaFuncSetAttribute(split_kernel<MODE, EASY>, cudaFuncAttributeMaxDynamicSharedMemorySize, Form<MODE>::DYNAMIC_BYTES));
        configured = true;
    }
    launch_kernel(split_kernel<MODE, EASY>, grid, THREADS, Form<MODE>::DYNAMIC_BYTES, stream, a);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

template <int MODE>
int32_t launch_mode(rtma_ctx* ctx, LinearArgs& a, void* planes, int cls, cudaStream_t stream) {
    if (MODE != WEIGHT_GRADIENT) {
        const int parts = a.w_stride ? a.G : 1, units = (a.d_out + 7) / 8;
        const int64_t ld = 8 * (int64_t)units, work = (int64_t)parts * a.d_in * units, blocks = ceil_div(work, 256);
        if (!make_tensor_map_16bit(&a.map_b, true, planes, 3 * (uint64_t)parts, a.d_in, a.d_out, ld, ld * a.d_in, MODE == FORWARD ? BK : a.BN,
                                   MODE == FORWARD ? 64 : 32, 3))
            return rtma_fail(ctx, RTMA_ERR_CUDA, "grouped product: no tensor map for %d matrices of %d x %d", parts, a.d_in, a.d_out);
        KernelScope ks(ctx, KC_WEIGHT_PREP, stream);
        launch_kernel(split_planes_kernel, (unsigned)(blocks < 16 * ctx->sm_count ? blocks : 16 * ctx->sm_count), 256, 0, stream,
                      static_cast<const float*>(a.B), a.w_stride, parts, a.d_in, a.d_out, a.vb, static_cast<__nv_bfloat16*>(planes));
        RTMA_LAUNCH_CHECK(ctx);
    }
    const int64_t tiles = a.tiles * a.m_tiles * a.n_tiles;
    const int64_t places = (int64_t)BLOCKS_PER_SM * ctx->sm_count;
    const unsigned grid = (unsigned)(tiles < places ? tiles : places);
    // operands on 16-byte boundaries with widths of whole 16 bytes are loaded without a case for every value
    const bool easy_a = a.va >= 16 && (MODE == INPUT_GRADIENT ? a.d_out : a.d_in) % 4 == 0, easy_b = a.vb >= 16 && a.d_out % 4 == 0;
    bool* configured = ctx->split_configured + 4 * MODE;
    KernelScope ks(ctx, cls, stream);
    if constexpr (MODE == WEIGHT_GRADIENT) {
        if (easy_b) return easy_a ? launch_form<MODE, 3>(ctx, a, grid, configured[3], stream) : launch_form<MODE, 2>(ctx, a, grid, configured[2], stream);
    }
    return easy_a ? launch_form<MODE, 1>(ctx, a, grid, configured[1], stream) : launch_form<MODE, 0>(ctx, a, grid, configured[0], stream);
}

}  // namespace

size_t split_planes_bytes(const LinearArgs& a) {
    return (size_t)3 * 2 * (a.w_stride ? a.G : 1) * a.d_in * ((a.d_out + 7) / 8 * 8);
}

int32_t launch_split(rtma_ctx* ctx, int mode, LinearArgs& a, void* planes, int cls, cudaStream_t stream) {
    const int64_t tiles = a.tiles * a.m_tiles * a.n_tiles;
    if (tiles >= (int64_t(1) << 30)) return rtma_fail(ctx, RTMA_ERR_OVERFLOW, "grouped product: %lld tiles", (long long)tiles);
    return mode == FORWARD ? launch_mode<FORWARD>(ctx, a, planes, cls, stream)
           : mode == INPUT_GRADIENT ? launch_mode<INPUT_GRADIENT>(ctx, a, planes, cls, stream)
                                    : launch_mode<WEIGHT_GRADIENT>(ctx, a, planes, cls, stream);
}
