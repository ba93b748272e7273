// The product of every part's rows with the part's own matrix, and its gradients:
//   forward  Y[r] = X[r] W_g + b_g        dx  dX[r] = dY[r] W_g^T        dw  dW_g = sum_r X[r]^T dY[r], db_g = sum_r dY[r]
// for the rows r of part g, on the tensor cores (tcgen05, accumulators in tensor memory).
//
// One kernel body serves all three: a tile is 128 x BN results, its operands are staged 64 deep in the contraction, each as 32-row
// slabs of 128 bytes per row in the 128-byte swizzle.  Rows that run along the contraction (X, dY; W in dx) make a K-major
// operand, rows across it (W forward; X and dY in dw) an MN-major one: both come from memory as they lie, nothing is transposed.
//
// The tensor cores truncate when they accumulate, so a long sum drifts towards zero by half a step per addition.  The weight
// gradient, whose result is fp32, therefore has its drain warps take the accumulator after every 128 rows and add it up in
// registers, rounded to nearest.  The column sums of dY are a product as well, with a left operand of ones: added up by the drain
// warps from shared memory they cost more than all else that these do (1M x 128 x 256 in fp16: 239 us; like this and with what came after it 161).
//
// This file: 16-bit rows (fp32 ones are in grouped_split.cu).  Three ways of loading:
//   COPIES  rows of an operand do not all lie on 16-byte boundaries: three or four groups of 4 warps with asynchronous copies of 8 or 4
//           bytes (or plain loads of 2), bulk-tensor loads for the other operand
//   BULK    rows on 16-byte boundaries: one thread with bulk-tensor loads
//   PAIR    the same on pairs of blocks (a cluster of two, MMAs of 256 rows) that bring half of the right operand each
// then 8 drain warps (a quarter of the lanes, every second 32 columns each) and one warp that issues the MMAs.
//
// What bounds it: up to 256 terms the rows' bytes (dx of 2M x 256 -> 256 in bf16 324 us, 6.3 TB/s).  Above that waiting for operands, though no
// unit is full: of 100,000 x 512 -> 512 on pairs (59 us under the profiler) the tensor pipes are busy for 43 %, the L2 cache for 34 %,
// memory for 35 % (500,000 rows 260 to 270 us, 1 PFLOP/s; 200,000 x 1024 -> 1024 356 us, 1.18).  The weight gradient reads each row of X and dY
// once per 128 columns of the other (1M x 256 x 256 in bf16 320 to 335 us), and shared memory, from which an MMA of 128 x 128 reads 128
// bytes a clock.  Rows off 16-byte boundaries: the copies (1M x 100 x 256 in fp16 200 to 230 us, 1M x 47 -> 90 in bf16 150); of that weight
// gradient with 500,000 rows shared memory's data path is busy for 50 %, instructions are issued in 48 % of the cycles, tensor pipes 28 %.
// Its kernel is the one here that spills: 256 bytes a thread at 72 registers (80 sums and 8 loaded values in a drain warp's lane).
#include <algorithm>

#include "grouped_rows.cuh"

RTMA_BOUNDS_TU()

namespace {

using namespace grouped;

constexpr int DW_WAVES = 2;                // tiles of a weight gradient for every block that runs at a time
constexpr int BIAS_ROWS = 1;               // of a slot: column sums of dY

// 32 columns (chunk `chunk` of the tile) of a warp's 32 rows (its quarter of the tile's) to the result.
template <class T, int MODE, class W, class OUT>
__device__ __forceinline__ void put_chunk(const LinearArgs& a, const W& w, OUT& outlet, const float (&v)[32], int quarter, int chunk, int lane) {
    typedef typename std::conditional<MODE == WEIGHT_GRADIENT, float, T>::type O;
    const int N = MODE == INPUT_GRADIENT ? a.d_in : MODE == FORWARD ? a.d_out : (int)a.ldo;  // (dw: the slots' rows are padded)
    const int c = w.n0 + 32 * chunk, cols = min(min(32, a.BN - 32 * chunk), N - c);
    const int rows = min(32, (MODE == WEIGHT_GRADIENT ? min(BM, a.d_in - w.m0) : w.rows) - 32 * quarter);
    if (cols <= 0 || rows <= 0) return;
    const int64_t row0 = (MODE == WEIGHT_GRADIENT ? (int64_t)w.row_tile * (a.d_in + BIAS_ROWS) + w.m0 : w.row0) + 32 * quarter;
    outlet.put(a, v, row0, c, rows, cols, c + cols == N && N % (16 / (int)sizeof(O)) == 0, static_cast<O*>(a.out) + row0 * a.ldo + c, a.ldo, lane);
}

template <class T, int MODE, int LOADING>
__device__ __forceinline__ void drain_role(const LinearArgs& a, Shared& sh, uint32_t slabs) {
    typedef Form<T, MODE, LOADING> F;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3, half = warp >> 2;
    typedef typename std::conditional<MODE == WEIGHT_GRADIENT, float, T>::type O;
    Outlet<O, F::OUT_SLABS> outlet{slabs + warp * F::OUT_BYTES};
    BiasHolder<T> bias{sh.bias + 128 * warp};
    const uint32_t tmem = sh.tmem_base + ((uint32_t)(32 * quarter) << 16);
    const int chunks = (a.BN + 31) / 32;
    typename F::Walks w;
    tc::RingAt acc;
    for (bool more = w.first(a, sh); more; more = w.next_tile(a, sh)) {
        if constexpr (MODE == WEIGHT_GRADIENT) {
            float total[2][32], sums[16];  // sums: of 16 columns, the same in every lane
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 32; ++j) total[i][j] = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) sums[j] = 0.f;
            const bool sums_wanted = a.db && w.m0 == 0 && 16 * warp < a.BN;
            for (int k0 = 0; k0 < w.k_end; k0 += F::ACC_STAGES * BK) {
                if (!wait_for<F::PAIRED>(&sh.acc_full[acc.s], acc.phase, sh, a.error_word)) return;
                __syncwarp();
                tc::tc_fence_after_sync();
                const uint32_t from = tmem + acc.s * F::ACC_COLUMNS;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (half + 2 * i < chunks) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float v[8];
                            tc::tmem_load_32x8(from + 32 * (half + 2 * i) + 8 * q, v);
#pragma unroll
                            for (int j = 0; j < 8; ++j) total[i][8 * q + j] += v[j];
                        }
                    }
                }
                if (sums_wanted) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float v[8];
                        tc::tmem_load_32x8(from + 128 + 16 * warp + 8 * q, v);
#pragma unroll
                        for (int j = 0; j < 8; ++j) sums[8 * q + j] += v[j];
                    }
                }
                tc::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sh.acc_empty[acc.s]);
                acc.advance(2);
            }
            if (sums_wanted && lane == 0) {
                float* to = static_cast<float*>(a.out) + ((int64_t)w.row_tile * (a.d_in + BIAS_ROWS) + a.d_in) * a.ldo + w.n0 + 16 * warp;
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (w.n0 + 16 * warp + j < a.d_out) to[j] = sums[j];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (half + 2 * i < chunks) put_chunk<T, MODE>(a, w, outlet, total[i], quarter, half + 2 * i, lane);
        } else {
            if (MODE == FORWARD && a.bias) bias.fetch(a, w.part, w.n0, half, 2, chunks, lane);
            if (!wait_for<F::PAIRED>(&sh.acc_full[acc.s], acc.phase, sh, a.error_word)) return;
            __syncwarp();
            tc::tc_fence_after_sync();
            for (int chunk = half; chunk < chunks; chunk += 2) {
                float v[32];
                tc::tmem_load_32x32(tmem + acc.s * F::ACC_COLUMNS + 32 * chunk, v);
                if (MODE == FORWARD && a.bias) bias.add(v, chunk >> 1);
                put_chunk<T, MODE>(a, w, outlet, v, quarter, chunk, lane);
            }
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {  // (a pair's warps all report to the first block)
                if constexpr (F::PAIRED) tc::mbar_arrive_remote(tc::leader_addr(&sh.acc_empty[acc.s]));
                else tc::mbar_arrive(&sh.acc_empty[acc.s]);
            }
            acc.advance(2);
        }
    }
    outlet.finish(lane);
}
template <class T, int MODE, int LOADING>
__global__ void __launch_bounds__(Form<T, MODE, LOADING>::THREADS, 1) linear_kernel(const __grid_constant__ LinearArgs a) {
    __shared__ Shared sh;
    linear_body<Form<T, MODE, LOADING>>(a, sh, [&](uint32_t slabs) { drain_role<T, MODE, LOADING>(a, sh, slabs); });
}
template <class T, int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Form<T, MODE, PAIR>::THREADS, 1) linear_pair_kernel(const __grid_constant__ LinearArgs a) {
    __shared__ Shared sh;
    linear_body<Form<T, MODE, PAIR>>(a, sh, [&](uint32_t slabs) { drain_role<T, MODE, PAIR>(a, sh, slabs); });
}

// The slots of every part added up in order.  A block takes 128 neighbouring places of a slot, its warps every eighth slot each; the
// row behind the weights is the bias's, whose partial sums lie in bias_rows rows (added up one after the other by one thread each they
// took 414 us for 16 parts; so, the kernel takes 10).
constexpr int REDUCE_THREADS = 256;
template <class O>
__global__ void __launch_bounds__(REDUCE_THREADS) linear_reduce_kernel(const __grid_constant__ LinearArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    __shared__ float4 red[8][32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.n ? *a.chunk_rows : 1, a.tiles, tile_start, warp_sums, a.span);
    const int part = blockIdx.y, lane = threadIdx.x & 31, share = threadIdx.x >> 5;
    const int64_t slot = (a.d_in + a.bias_rows) * a.ldo, i = ((int64_t)blockIdx.x * 32 + lane) * 4;
    const int row = (int)(i / a.ldo), col = (int)(i - row * a.ldo);
    const int t0 = tile_start[part], t1 = tile_start[part + 1];
    const float* p = static_cast<const float*>(a.out) + t0 * slot + i;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float4 v) {
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
    };
    if (row < a.d_in) {
#pragma unroll 4
        for (int t = share; t < t1 - t0; t += 8) add(*reinterpret_cast<const float4*>(p + t * slot));
    } else if (row == a.d_in) {
#pragma unroll 4
        for (int j = share; j < (t1 - t0) * a.bias_rows; j += 8) add(*reinterpret_cast<const float4*>(p + j / a.bias_rows * slot + j % a.bias_rows * a.ldo));
    }
    red[share][lane] = s;
    __syncthreads();
    if (share || row > a.d_in || (row == a.d_in && !a.db)) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) add(red[k][lane]);
    const int run = col / a.fold, c = col - run * a.fold, real = a.d_out / a.fold * a.fold_real;
    O* to = (row < a.d_in ? static_cast<O*>(a.dW) + part * a.dw_stride + (int64_t)row * real : static_cast<O*>(a.db) + part * a.db_stride) + run * a.fold_real + c;
    const int left = min(a.fold_real - c, a.d_out - col);
    if (left > 0) to[0] = from_f32<O>(s.x);
    if (left > 1) to[1] = from_f32<O>(s.y);
    if (left > 2) to[2] = from_f32<O>(s.z);
    if (left > 3) to[3] = from_f32<O>(s.w);
}

// Columns in equal tiles of a multiple of 16.
void cut_columns(LinearArgs& a, int N, int widest) {
    a.n_tiles = (int)ceil_div(N, widest);
    a.BN = (int)ceil_div(ceil_div(N, a.n_tiles), 16) * 16;
    a.n_tiles = (int)ceil_div(N, a.BN);
}

// A few us: 16-bit matrices whose rows do not lie on 16-byte boundaries -> [part][d_in][ld] that do (ld: d_out rounded up to 8)
__global__ void __launch_bounds__(256) pad_matrices_kernel(const __half* __restrict__ W, int64_t w_stride, int parts, int d_in, int d_out, int granule,
                                                           __half* __restrict__ out) {
    wait_for_kernel_before();
    const int units = (d_out + 7) / 8;
    const int64_t total = (int64_t)parts * d_in * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / units, part = row / d_in;
        const int u = (int)(i - row * units);
        Eight<__half> x;
        x.load(W + part * w_stride + (row - part * d_in) * d_out + 8 * u, min(8, d_out - 8 * u), granule);
        *reinterpret_cast<uint4*>(out + 8 * i) = x.w[0];
    }
}

int32_t pad_matrices(rtma_ctx* ctx, LinearArgs& a, cudaStream_t stream) {
    const int parts = a.w_stride ? a.G : 1, units = (a.d_out + 7) / 8;
    const int64_t blocks = ceil_div((int64_t)parts * a.d_in * units, 256);
    KernelScope ks(ctx, KC_WEIGHT_PREP, stream);
    launch_kernel(pad_matrices_kernel, (unsigned)std::min<int64_t>(blocks, 16 * ctx->sm_count), 256, 0, stream, static_cast<const __half*>(a.B), a.w_stride,
                  parts, a.d_in, a.d_out, a.vb, reinterpret_cast<__half*>(ctx->arena));
    RTMA_LAUNCH_CHECK(ctx);
    a.B = ctx->arena;
    a.ldb = 8 * units;
    a.w_stride = a.w_stride ? a.d_in * a.ldb : 0;
    a.vb = 16;
    return RTMA_OK;
}

template <class T, int MODE, int LOADING>
int32_t launch_form(rtma_ctx* ctx, const LinearArgs& a, unsigned grid, bool& configured, cudaStream_t stream) {
    void (*kernel)(LinearArgs);
    if constexpr (LOADING == PAIR) kernel = linear_pair_kernel<T, MODE>;
    else kernel = linear_kernel<T, MODE, LOADING>;
    if (!configured) {
        RTMA_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Form<T, MODE, LOADING>::DYNAMIC_BYTES));
        configured = true;
    }
    launch_kernel(kernel, grid, Form<T, MODE, LOADING>::THREADS, Form<T, MODE, LOADING>::DYNAMIC_BYTES, stream, a);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

// Which operands bulk-tensor loads can fetch (1: the left one, 2: the right one); sets up their maps.
template <int MODE>
int bulk_maps(LinearArgs& a, bool bf16, bool pair) {
    int in_bulk = 0;
    if (a.va >= 16) {
        const bool ok = MODE == WEIGHT_GRADIENT ? make_tensor_map_16bit(&a.map_a, bf16, a.A, 1, a.n, a.d_in, a.lda, a.n * a.lda, BK)
                                                : make_tensor_map_16bit(&a.map_a, bf16, a.A, 1, a.n, MODE == FORWARD ? a.d_in : a.d_out, a.lda, a.n * a.lda, BM);
        in_bulk |= ok ? 1 : 0;
    }
    if (a.vb >= 16 && a.w_stride >= 0) {
        const bool ok = MODE == WEIGHT_GRADIENT ? make_tensor_map_16bit(&a.map_b, bf16, a.B, 1, a.n, a.d_out, a.ldb, a.n * a.ldb, BK)
                                                : make_tensor_map_16bit(&a.map_b, bf16, a.B, a.w_stride ? a.G : 1, a.d_in, a.d_out, a.ldb,
                                                                        a.w_stride ? a.w_stride : a.d_in * a.ldb, MODE == FORWARD ? BK : pair ? a.BN / 2 : a.BN);
        in_bulk |= ok ? 2 : 0;
    }
    return in_bulk;
}

template <int MODE>
int32_t launch_linear(rtma_ctx* ctx, int32_t dtype, LinearArgs& a, int cls, cudaStream_t stream) {
    a.error_word = ctx->error_word;
    if (dtype == RTMA_F32) return launch_split(ctx, MODE, a, MODE == WEIGHT_GRADIENT ? nullptr : ctx->arena, cls, stream);
    const int64_t tiles = a.tiles * a.m_tiles * a.n_tiles;
    if (tiles >= (int64_t(1) << 30)) return rtma_fail(ctx, RTMA_ERR_OVERFLOW, "grouped product: %lld tiles", (long long)tiles);
    const unsigned grid = (unsigned)(tiles < ctx->sm_count ? tiles : ctx->sm_count);
    bool* configured = ctx->linear_configured + MODE * 4;
    KernelScope ks(ctx, cls, stream);
    const bool bf16 = dtype == RTMA_BF16;
    // Pairs of blocks where the contraction is deep: each then brings half of the right operand, which comes from the L2 cache again for
    // every tile (bf16, alone / in pairs: 500,000 x 512 -> 512 285 / 270 us, 30,000 rows 35 / 27; 1M x 256 -> 256 181 / 170, 30,000 rows
    // 17 / 14).  Short contractions are drains, which a pair's blocks wait for together: 1M x 64 -> 256 123 / 133.  A pair's block brings 128
    // columns, so tiles of other widths (384 columns are two of 192, 600 three of 208) never pair.
    bool pair = false;
    if constexpr (MODE != WEIGHT_GRADIENT) pair = a.BN == 256 && (MODE == FORWARD ? a.d_in : a.d_out) >= 256 && tiles >= ctx->sm_count;
    a.in_bulk = bulk_maps<MODE>(a, bf16, pair);
    if constexpr (MODE != WEIGHT_GRADIENT) {
        if (pair && a.in_bulk == 3) {
            a.tile_rows = 2 * BM;
            a.tiles = a.n / a.tile_rows + a.G;
            const int64_t blocks = 2 * a.tiles * a.n_tiles, places = ctx->sm_count & ~1;
            bool* once = ctx->linear_configured + 12 + (MODE == FORWARD ? 0 : 2);
            return bf16 ? launch_form<__nv_bfloat16, MODE, PAIR>(ctx, a, (unsigned)std::min(blocks, places), once[0], stream)
                        : launch_form<__half, MODE, PAIR>(ctx, a, (unsigned)std::min(blocks, places), once[1], stream);
        }
        if (pair) a.in_bulk = 0;  // (the right operand's map is one for pairs)
    }
    if (a.in_bulk == 3)
        return bf16 ? launch_form<__nv_bfloat16, MODE, BULK>(ctx, a, grid, configured[0], stream) : launch_form<__half, MODE, BULK>(ctx, a, grid, configured[1], stream);
    return bf16 ? launch_form<__nv_bfloat16, MODE, COPIES>(ctx, a, grid, configured[2], stream) : launch_form<__half, MODE, COPIES>(ctx, a, grid, configured[3], stream);
}

int32_t check_linear(rtma_ctx* ctx, const char* who, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out) {
    RTMA_TRY(check_parts(ctx, who, n, G, offsets));
    if (dtype < RTMA_F32 || dtype > RTMA_F16) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: dtype=%d", who, dtype);
    if (d_in < 1 || d_out < 1 || d_in > RTMA_MAX_WIDTH || d_out > RTMA_MAX_WIDTH)
        return rtma_fail(ctx, RTMA_ERR_UNSUPPORTED, "%s: %d x %d outside [1,%d]", who, d_in, d_out, RTMA_MAX_WIDTH);
    return RTMA_OK;
}

}  // namespace

int32_t grouped_rows(rtma_ctx* ctx, const char* who, bool transposed, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                     const void* A, int64_t lda, const void* W, int64_t w_stride, const void* b, int64_t b_stride, void* out, int64_t ldo, size_t* scratch,
                     cudaStream_t stream) {
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_linear(ctx, who, dtype, n, G, offsets, d_in, d_out));
    if (scratch) *scratch = 0;
    if (n == 0) return RTMA_OK;
    if (!A || !W || !out) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: null pointer", who);
    const int K = transposed ? d_out : d_in, N = transposed ? d_in : d_out;
    if (lda < K || ldo < N) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: rows of %d and %d values lie closer than that", who, K, N);
    if (A == out) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: the result must not overlap the rows", who);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    const size_t es = row_type_bytes(dtype);
    LinearArgs a{};
    a.offsets = offsets; a.n = n; a.G = G; a.span = 1;
    a.tile_rows = BM;
    a.tiles = n / BM + G;
    a.m_tiles = 1;
    cut_columns(a, N, dtype == RTMA_F32 ? SPLIT_COLUMNS : 256);
    a.d_in = d_in; a.d_out = d_out;
    a.A = A; a.lda = lda; a.B = W; a.ldb = d_out; a.w_stride = w_stride; a.bias = b; a.bias_stride = b_stride;
    a.bias_overlaps = G > 1 && b_stride != 0 && b_stride < d_out && b_stride > -d_out;
    a.va = row_granule(A, lda, es);
    a.vb = std::min(row_granule(W, d_out, es), row_granule(nullptr, w_stride, es));
    a.out = out; a.ldo = ldo;
    a.go = row_granule(out, ldo, es);
    a.vo = dtype != RTMA_F32 && a.go >= 16 && make_store_map(&a.map_o, dtype, out, n, N, ldo);
    // Matrices with rows on other boundaries are laid out on 16-byte ones first if a block would copy them more than once: 1M x 256 -> 47
    // in bf16 208 -> 126 us, its dx 261 -> 175; 32,000 rows 16.5 -> 15.1 and 17.9 -> 14.9; for a tile or less per block it is a launch more.
    const bool pad = dtype != RTMA_F32 && a.vb < 16 && a.tiles > ctx->sm_count;
    const size_t padded = (size_t)2 * (w_stride ? G : 1) * d_in * ceil_div(d_out, 8) * 8;
    const size_t bytes = dtype == RTMA_F32 ? split_planes_bytes(a) : pad ? padded : 0;
    if (scratch) {
        *scratch = bytes;
        return RTMA_OK;
    }
    RTMA_TRY(prepare_row_call(ctx, bytes, stream));
    if (pad) RTMA_TRY(pad_matrices(ctx, a, stream));
    return transposed ? launch_linear<INPUT_GRADIENT>(ctx, dtype, a, KC_GEMM_DGRAD, stream) : launch_linear<FORWARD>(ctx, dtype, a, KC_GEMM_FWD, stream);
}

int32_t grouped_dw(rtma_ctx* ctx, const char* who, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out, const void* X,
                   int64_t ldx, const void* dY, int64_t lddy, int fold, int fold_real, int32_t out_dtype, void* dW, int64_t dw_stride, void* db, int64_t db_stride, size_t* scratch,
                   cudaStream_t stream) {
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_linear(ctx, who, dtype, n, G, offsets, d_in, d_out));
    if (!dW || (n > 0 && (!X || !dY))) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: null pointer", who);
    if (ldx < d_in || lddy < d_out) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: rows of %d and %d values lie closer than that", who, d_in, d_out);
    const int real_out = d_out / fold * fold_real;
    const int64_t weights = (int64_t)d_in * real_out;
    const bool shared = G > 1 && dw_stride == 0;
    if (G > 1 && db && (db_stride == 0) != shared)
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: either both gradients are one for all parts or neither", who);
    if (G > 1 && !shared && ((dw_stride < weights && dw_stride > -weights) || (db && db_stride < real_out && db_stride > -real_out)))
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: gradients of the parts overlap", who);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    LinearArgs a{};
    a.offsets = offsets; a.n = n;
    a.G = shared ? 1 : G;
    a.span = shared ? G : 1;
    a.m_tiles = (int)ceil_div(d_in, BM);
    a.bias_rows = dtype == RTMA_F32 ? SPLIT_BIAS_ROWS : BIAS_ROWS;
    cut_columns(a, d_out, dtype == RTMA_F32 ? SPLIT_DW_COLUMNS : 128);
    // DW_WAVES tiles for every block that runs at a time (a chunk per part at least), of 256 rows or more
    const int64_t places = (int64_t)ctx->sm_count * (dtype == RTMA_F32 ? SPLIT_BLOCKS_PER_SM : 1);
    a.tile_rows = 256;
    a.tiles = std::min(std::max<int64_t>(a.G, DW_WAVES * places / ((int64_t)a.m_tiles * a.n_tiles)), n / a.tile_rows + a.G);
    const size_t es = row_type_bytes(dtype);
    a.d_in = d_in; a.d_out = d_out;
    a.A = X; a.lda = ldx; a.B = dY; a.ldb = lddy;
    a.va = row_granule(X, ldx, es);
    a.vb = row_granule(dY, lddy, es);
    a.dW = dW; a.dw_stride = dw_stride; a.db = db; a.db_stride = db_stride;
    a.fold = fold; a.fold_real = fold_real;
    a.ldo = ceil_div(d_out, 8) * 8;
    a.go = 32;
    const int64_t slot_rows = a.tiles * (d_in + a.bias_rows);
    const size_t bytes = 256 + sizeof(float) * slot_rows * a.ldo;
    if (scratch) {
        *scratch = bytes;
        return RTMA_OK;
    }
    RTMA_TRY(prepare_row_call(ctx, bytes, stream));
    a.chunk_rows = reinterpret_cast<int32_t*>(ctx->arena);
    a.out = ctx->arena + 256;
    a.vo = dtype != RTMA_F32 && slot_rows < (int64_t(1) << 31) && make_store_map(&a.map_o, RTMA_F32, a.out, slot_rows, a.ldo, a.ldo);
    if (n > 0) RTMA_TRY(launch_linear<WEIGHT_GRADIENT>(ctx, dtype, a, KC_GEMM_WGRAD, stream));
    {
        KernelScope ks(ctx, KC_REDUCE_SGD, stream);
        void (*reduce)(LinearArgs) = out_dtype == RTMA_F32 ? linear_reduce_kernel<float> : out_dtype == RTMA_BF16 ? linear_reduce_kernel<__nv_bfloat16> : linear_reduce_kernel<__half>;
        launch_kernel(reduce, dim3((unsigned)ceil_div((d_in + 1) * a.ldo, 128), (unsigned)a.G), REDUCE_THREADS, 0, stream, a);
    }
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

extern "C" int32_t rtma_grouped_linear(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                                       const void* X, int64_t ldx, const void* W, int64_t w_stride, const void* b, int64_t b_stride, void* Y,
                                       int64_t ldy, void* stream) {
    return grouped_rows(ctx, "rtma_grouped_linear", false, dtype, n, G, offsets, d_in, d_out, X, ldx, W, w_stride, b, b_stride, Y, ldy, nullptr,
                        static_cast<cudaStream_t>(stream));
}

extern "C" int32_t rtma_grouped_linear_dx(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                                          const void* dY, int64_t lddy, const void* W, int64_t w_stride, void* dX, int64_t lddx, void* stream) {
    return grouped_rows(ctx, "rtma_grouped_linear_dx", true, dtype, n, G, offsets, d_in, d_out, dY, lddy, W, w_stride, nullptr, 0, dX, lddx, nullptr,
                        static_cast<cudaStream_t>(stream));
}

extern "C" int32_t rtma_grouped_linear_dw(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                                          const void* X, int64_t ldx, const void* dY, int64_t lddy, float* dW, int64_t dw_stride, float* db,
                                          int64_t db_stride, void* stream) {
    return grouped_dw(ctx, "rtma_grouped_linear_dw", dtype, n, G, offsets, d_in, d_out, X, ldx, dY, lddy, d_out, d_out, RTMA_F32, dW, dw_stride, db, db_stride, nullptr,
                      static_cast<cudaStream_t>(stream));
}
