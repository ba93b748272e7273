// Layers over the rows of many parts, on the tensor cores:
//   Y[r] = R[r] + act(X[r] W_g + b_g)                          gated: H[r] = R[r] + act(X[r] V_g + c_g) * (X[r] U_g + d_g)
// for the rows r of part g, W_g = [V_g | U_g] in a gated layer, and the first step of their gradients,
//   dZ[r] = dY[r] act'(Z[r])                                   gated: dZ[r] = [dH u act'(v) | dH act(v)]
// with Z = X W + b worked out again from the inputs.  Kept from the forward pass, Z would cost a write there and a read here: of 16-bit rows
// that is more than the product as long as the contraction has fewer than about 600 terms, and nothing of the forward pass has to be kept.
// dX = dZ W^T and dW = X^T dZ are products of their own, and dZ, an operand of these, is rounded to the rows' type.
//
// The product stays in tensor memory and goes through the layer in the registers of the warps that drain it.  A tile of a gated layer has the same columns
// of both matrices, so that a lane finds both factors of a result in its own row.  Rows off 16-byte boundaries, and matrices whose rows lie so, are laid
// out on such boundaries first: one way through the products for all rows.
//
// This file: the calls and what is laid out.  The layers' kernels: layer_pairs.cuh (16-bit rows), layer_f32.cu; the weight gradients': layer_wgrad.cu; dX of
// 16-bit rows is a call of grouped_linear.cu.
#include <algorithm>

#include "layer.cuh"

RTMA_BOUNDS_TU()

namespace {

using namespace grouped;

constexpr int PAIR_ROWS = 2 * PAIR_BM;  // of a pair's tile

// 16-bit rows on any boundary -> rows on 16-byte ones, zeros behind each up to a multiple of 8 values.  Row r lies at src + (r / group) *
// group_stride + (r % group) * ld.
struct AlignJob {
    const uint16_t* src;
    uint16_t* dst;
    int64_t rows, group, group_stride, ld;
    int d, granule;
};
struct AlignArgs {
    AlignJob job[3];
};
constexpr int ALIGN_BYTES = 16384;

// A block brings neighbouring rows as the 16-byte words that they lie in, and cuts them up in shared memory while the next ones come (200,000 x 100 in
// fp16 24 us; 300,000 x 100 and x 47 37 us, 4.8 TB/s: instructions, of which they issue 64 % of what they can).  Copied by the products for every
// tile of columns again, such rows cost more than the products: 200,000 x 100 -> 2 x 266 222 us, like this 81 and 24.
__global__ void __launch_bounds__(256) align_rows_kernel(const __grid_constant__ AlignArgs args) {
    __shared__ uint4 words[ALIGN_BYTES / 16 + 258];  // (a row's last words are read beyond it, and dropped)
    wait_for_kernel_before();
    const AlignJob& a = args.job[blockIdx.y];
    if (!a.rows) return;
    const int units = (a.d + 7) / 8;
    const int together = a.ld <= 2 * (int64_t)a.d && a.ld * 2 <= ALIGN_BYTES ? (int)min(a.group, ALIGN_BYTES / (a.ld * 2)) : 0;  // rows at a time
    if (!together) {
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.rows * units; i += (int64_t)gridDim.x * 256) {
            const int64_t row = i / units, part = row / a.group;
            const int u = (int)(i - row * units);
            Eight<__half> x;
            x.load(reinterpret_cast<const __half*>(a.src) + part * a.group_stride + (row - part * a.group) * a.ld + 8 * u, min(8, a.d - 8 * u), a.granule);
            *reinterpret_cast<uint4*>(a.dst + 8 * i) = x.w[0];
        }
        return;
    }
    const int64_t per_group = (a.group + together - 1) / together, all = a.rows / a.group * per_group;
    constexpr int LOADS = ALIGN_BYTES / 16 / 256 + 1;
    struct Chunk {
        int64_t row0;  // of all rows
        int rows;
        uintptr_t from, to, base;
    };
    auto chunk = [&](int64_t c) {
        const int64_t part = c / per_group, first = (c - part * per_group) * together;
        Chunk k;
        k.row0 = part * a.group + first;
        k.rows = (int)min((int64_t)together, a.group - first);
        k.from = reinterpret_cast<uintptr_t>(a.src + part * a.group_stride + first * a.ld);
        k.to = k.from + 2 * ((k.rows - 1) * a.ld + a.d);
        k.base = k.from & ~(uintptr_t)15;
        return k;
    };
    uint4 x[LOADS];
    auto bring = [&](const Chunk& k) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uintptr_t p = k.base + 16 * (uintptr_t)(threadIdx.x + 256 * i);
            if (p >= k.from && p + 16 <= k.to) {
                x[i] = *reinterpret_cast<const uint4*>(p);
            } else if (p < k.to) {  // a word that is not the rows' alone
                uint32_t w[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const uintptr_t e = p + 4 * h;
                    const uint32_t lo = e >= k.from && e < k.to ? *reinterpret_cast<const uint16_t*>(e) : 0u, hi = e + 2 >= k.from && e + 2 < k.to ? *reinterpret_cast<const uint16_t*>(e + 2) : 0u;
                    w[h] = lo | hi << 16;
                }
                x[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    };
    int64_t c = blockIdx.x;
    if (c >= all) return;
    Chunk now = chunk(c);
    bring(now);
    const int ld = (int)a.ld, rows_on = 256 / units, on = 256 - rows_on * units;
    for (;;) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if (now.base + 16 * (uintptr_t)(threadIdx.x + 256 * i) < now.to) words[threadIdx.x + 256 * i] = x[i];
        __syncthreads();
        const Chunk these = now;
        c += gridDim.x;
        const bool more = c < all;
        if (more) {  // the next ones are on their way while these are cut up
            now = chunk(c);
            bring(now);
        }
        // 16 bytes a thread: two words, of which the row's place in them says which five halves are wanted
        const int shift = (int)(these.from - these.base) / 2;
        uint4* out = reinterpret_cast<uint4*>(a.dst) + these.row0 * units;
        int row = threadIdx.x / units, unit = threadIdx.x - row * units;
        for (int i = threadIdx.x; i < these.rows * units; i += 256) {
            const int e = shift + row * ld + 8 * unit, valid = a.d - 8 * unit;
            const uint4 lo = words[e >> 3], hi = words[(e >> 3) + 1];
            uint32_t w[7] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z};
            if (e & 4) {
                w[0] = w[2]; w[1] = w[3]; w[2] = w[4]; w[3] = w[5]; w[4] = w[6]; w[5] = hi.w;
            }
#pragma unroll
            for (int k = 0; k < 5; ++k) w[k] = e & 2 ? w[k + 1] : w[k];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                w[k] = __funnelshift_r(w[k], w[k + 1], 16 * (e & 1));
                if (valid < 2 * k + 2) w[k] = valid == 2 * k + 1 ? w[k] & 0xFFFFu : 0u;
            }
            out[i] = make_uint4(w[0], w[1], w[2], w[3]);
            row += rows_on;
            unit += on;
            if (unit >= units) {
                unit -= units;
                ++row;
            }
        }
        if (!more) return;
        __syncthreads();
    }
}

constexpr int MOST_PLACES = 256;  // pairs of blocks on a GPU at most

struct SumsArgs {
    const int64_t* offsets;
    int64_t n, tile_rows, tiles;
    int G, places, n_tiles, columns;  // columns: 0 if their sums are not wanted
    int width, real_width;            // of one of dZ's halves, with and without what was rounded up
    const float *column_slots, *slope_slots;
    int64_t slots_up;  // as LayerArgs'
    int groups_log;
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
constexpr int SUMS_THREADS = 512;
template <class O>
__global__ void __launch_bounds__(SUMS_THREADS) layer_sums_kernel(const __grid_constant__ SumsArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32], place_start[MOST_PLACES + 1];
    __shared__ double red[SUMS_THREADS];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int64_t tiles = tile_start[a.G];
    for (int i = threadIdx.x; i <= a.places; i += SUMS_THREADS) place_start[i] = (int)(tiles * i / a.places);
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool of_slope = (int)blockIdx.x * 32 >= a.columns, shared = of_slope ? a.slope_shared : a.shared;
    if ((int)blockIdx.y > 0 && shared) return;
    const int column = 32 * blockIdx.x + lane, first = shared ? 0 : blockIdx.y, last = shared ? a.G : first + 1;
    double s = 0.0;
    for (int part = first; part < last; ++part) {
        const int from = tile_start[part], to = tile_start[part + 1];
        if (from == to) continue;
        // the places whose tiles are among the part's; those without tiles have left no slot
        int i = (int)((int64_t)from * a.places / tiles), end;
        while (place_start[i + 1] <= from) ++i;
        for (end = i + 1; end < a.places && place_start[end] < to;) ++end;
        if (!of_slope) {  // eight warps for the sums of a slot, every second slot
            const float* p = a.column_slots + (8 * (int64_t)(i + part) + (warp & 7)) * a.columns + min(column, a.columns - 1);
#pragma unroll 4
            for (int x = warp >> 3; x < (end - i) << a.groups_log; x += SUMS_THREADS / 256) {
                const int k = x >> a.groups_log, group = x - (k << a.groups_log);
                const float v = p[(group * a.slots_up + 8 * (int64_t)k) * a.columns];
                s += place_start[i + k] != place_start[i + k + 1] ? v : 0.f;
            }
        } else {
            const int per = 32 * a.n_tiles;
            for (int k = threadIdx.x; k < (end - i) * per; k += SUMS_THREADS) {
                const int at = i + k / per;
                if (place_start[at] != place_start[at + 1]) s += a.slope_slots[(int64_t)(i + part) * per + k];
            }
        }
    }
    red[threadIdx.x] = s;
    __syncthreads();
    if (warp) return;
#pragma unroll 8
    for (int k = 1; k < SUMS_THREADS / 32; ++k) s += red[32 * k + lane];
    if (!of_slope) {
        if (column < a.columns && a.place_of(column) >= 0) static_cast<O*>(a.db)[blockIdx.y * a.db_stride + a.place_of(column)] = from_f32<O>((float)s);
    } else {
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) a.dslope[blockIdx.y * a.dslope_stride] = (float)s;
    }
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

// What is laid out first, where in the scratch, and the tiles.  Rows that lie on 16-byte boundaries are used where they are.
struct Plan {
    bool f32, lay_x, lay_side, lay_w;
    int halves, up;               // up: columns from one of the laid out matrices to the other
    int ld, ldt;                  // fp32: of the planes of the matrices, and of their transposes
    size_t x_at, side_at, w_at, wt_at, end;
    int n_tiles, half, places;
    int64_t tiles;
};

int columns_of(const rtma_layer_desc* d) { return (d->d_out + 7) / 8 * 8; }

// Pairs of blocks on N columns: equal tiles of 256 at most in steps of `step`.
void cut_tiles(const rtma_ctx* ctx, int N, int step, int64_t tiles, int& n_tiles, int& half, int& places) {
    n_tiles = (int)ceil_div(N, 256);
    half = (int)ceil_div(ceil_div(N, n_tiles), step) * step / 2;
    n_tiles = (int)ceil_div(N, 2 * half);
    places = (int)std::min<int64_t>(std::min(MOST_PLACES, std::max(1, ctx->sm_count / 2 / n_tiles)), tiles);
}

// gradient: dZ and what it is multiplied by have columns_of the layer's width.
Plan make_plan(const rtma_ctx* ctx, const rtma_layer_desc* d, int64_t n, int32_t G, const void* X, int64_t ldx, const void* W, const void* side, int64_t lds, bool gradient) {
    Plan p{};
    const bool plain = !d->gated && d->act == RTMA_ACT_NONE;
    const size_t es = row_type_bytes(d->dtype);
    const int64_t parts = d->w_stride ? G : 1;
    const int width = gradient && !plain ? columns_of(d) : d->d_out;
    p.f32 = d->dtype == RTMA_F32;
    p.halves = d->gated ? 2 : 1;
    p.lay_x = row_granule(X, ldx, es) < 16;
    // (16-bit: a gradient that is dZ itself is an operand whole, and what lies behind its rows is not zero)
    p.lay_side = side && (row_granule(side, lds, es) < 16 || (!p.f32 && gradient && plain && d->d_out % 8));
    ArenaCursor room(nullptr);
    p.x_at = room.used;
    if (p.lay_x) room.take<char>(es * n * ((d->d_in + 7) / 8 * 8));
    p.side_at = room.used;
    if (p.lay_side) room.take<char>(es * n * columns_of(d));
    p.w_at = p.wt_at = room.used;
    p.tiles = n / PAIR_ROWS + G;
    if (p.f32) {
        p.up = plain ? d->d_out : columns_of(d);
        p.ld = d->gated ? (width + 31) / 32 * 64 : (width + 7) / 8 * 8;
        p.ldt = (d->d_in + 7) / 8 * 8;
        room.take<uint16_t>(3 * (size_t)parts * d->d_in * p.ld);
        p.wt_at = room.used;
        if (gradient) room.take<uint16_t>(3 * (size_t)parts * p.halves * p.up * p.ldt);
        cut_tiles(ctx, p.ld, d->gated ? 64 : 32, p.tiles, p.n_tiles, p.half, p.places);
    } else {
        p.lay_w = row_granule(W, (int64_t)p.halves * d->d_out, 2) < 16 || row_granule(nullptr, d->w_stride, 2) < 16 || d->w_stride < 0 || (d->d_out % 8 && (d->gated || gradient));
        p.up = p.lay_w ? columns_of(d) : d->d_out;
        if (p.lay_w) room.take<uint16_t>((size_t)parts * d->d_in * p.halves * p.up);
        const int columns = gradient ? columns_of(d) : d->d_out;
        if (d->gated) {  // as many of either matrix
            cut_tiles(ctx, 2 * columns, 32, p.tiles, p.n_tiles, p.half, p.places);
            p.n_tiles = (int)ceil_div(columns, p.half);
            p.places = (int)std::min<int64_t>(std::min(MOST_PLACES, std::max(1, ctx->sm_count / 2 / p.n_tiles)), p.tiles);
        } else {
            cut_tiles(ctx, columns, 32, p.tiles, p.n_tiles, p.half, p.places);
        }
    }
    p.end = room.used;
    return p;
}

// Lays out what has to be and points X, side and W there.
int32_t lay_out_rows(rtma_ctx* ctx, const Plan& p, const rtma_layer_desc* d, int64_t n, int32_t G, const void*& X, int64_t& ldx, const void*& side, int64_t& lds, const void*& W,
                     int64_t& w_stride, cudaStream_t stream) {
    if (!p.lay_x && !p.lay_side && !p.lay_w) return RTMA_OK;
    const int values = (int)row_type_bytes(d->dtype) / 2;  // 16-bit ones in one of the rows'
    AlignArgs args{};
    auto job = [&](AlignJob& j, const void* src, size_t at, int64_t rows, int64_t group, int64_t group_stride, int64_t ld, int width) {
        j.src = static_cast<const uint16_t*>(src);
        j.dst = reinterpret_cast<uint16_t*>(ctx->arena + at);
        j.rows = rows; j.group = group; j.group_stride = group_stride; j.ld = ld; j.d = width;
        j.granule = std::min(row_granule(src, ld, 2), row_granule(nullptr, group_stride, 2));
    };
    auto rounded = [&](int width) { return (int64_t)((values * width + 7) / 8 * 8) / values; };
    if (p.lay_x) {
        job(args.job[0], X, p.x_at, n, n, 0, values * ldx, values * d->d_in);
        X = args.job[0].dst;
        ldx = rounded(d->d_in);
    }
    if (p.lay_side) {
        job(args.job[1], side, p.side_at, n, n, 0, values * lds, values * d->d_out);
        side = args.job[1].dst;
        lds = rounded(d->d_out);
    }
    if (p.lay_w) {
        const int64_t rows = (int64_t)d->d_in * p.halves;
        job(args.job[2], W, p.w_at, (w_stride ? G : 1) * rows, rows, w_stride, d->d_out, d->d_out);
        W = args.job[2].dst;
        w_stride = w_stride ? rows * p.up : 0;
    }
    int64_t blocks = 1;
    for (const AlignJob& j : args.job) blocks = std::max(blocks, ceil_div(j.rows * ((j.d + 7) / 8), 1024));
    KernelScope ks(ctx, KC_WEIGHT_PREP, stream);
    launch_kernel(align_rows_kernel, dim3((unsigned)std::min<int64_t>(blocks, 8 * ctx->sm_count), 3), 256, 0, stream, args);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

// What all kernels of a layer take.  width: columns of the result (of each of its halves).
LayerArgs layer_args(const rtma_ctx* ctx, const Plan& p, const rtma_layer_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx, const void* W,
                     int64_t w_stride, const void* b, const float* slope, const void* side, int64_t lds, void* out, int64_t ldo, int width) {
    const size_t es = row_type_bytes(d->dtype);
    LayerArgs a{};
    a.error_word = ctx->error_word;
    a.offsets = offsets; a.n = n; a.G = G; a.span = 1;
    a.m_tiles = 1;
    a.tile_rows = PAIR_ROWS; a.tiles = p.tiles;
    a.n_tiles = p.n_tiles; a.half = p.half; a.places = p.places;
    a.d_in = d->d_in; a.d_out = a.bias_up = a.bias_width = d->d_out;
    a.width = width;
    a.up = p.up;
    a.A = X; a.lda = ldx; a.B = p.f32 ? ctx->arena + p.w_at : W; a.ldb = p.f32 ? p.ld : p.halves * (int64_t)p.up; a.w_stride = w_stride;
    a.bias = b; a.bias_stride = d->b_stride;
    a.act = d->act;
    a.slope = d->act == RTMA_ACT_PRELU ? slope : nullptr; a.slope_stride = d->slope_stride;
    a.side = side; a.lds = lds;
    a.out = out; a.ldo = ldo;
    a.go = row_granule(out, ldo, es);
    return a;
}

// The layer's kernel; columns: of the whole result.
int32_t launch_layer(rtma_ctx* ctx, LayerArgs& a, const Plan& p, const rtma_layer_desc* d, bool gradient, int columns, cudaStream_t stream) {
    const bool bf16 = d->dtype == RTMA_BF16, gated = d->gated != 0;
    const unsigned grid = 2u * p.places * p.n_tiles;
    a.vo = a.go >= 16 && make_store_map(&a.map_o, d->dtype, a.out, a.n, columns, a.ldo);
    if (p.f32) return launch_layer_f32(ctx, a, gated, gradient, KC_GEMM_FWD, grid, stream);
    if (!make_tensor_map_16bit(&a.map_b, bf16, a.B, a.w_stride ? a.G : 1, a.d_in, a.ldb, a.ldb, a.w_stride ? a.w_stride : a.d_in * a.ldb, 64) ||
        !make_tensor_map_16bit(&a.map_a, bf16, a.A, 1, a.n, a.d_in, a.lda, a.n * a.lda, PAIR_ROWS / 2) ||
        (a.side && !make_store_map(&a.map_side, d->dtype, a.side, a.n, d->d_out, a.lds)))
        return rtma_fail(ctx, RTMA_ERR_CUDA, "grouped layer: no tensor map for rows of %d and %d values", a.d_in, d->d_out);
    KernelScope ks(ctx, KC_GEMM_FWD, stream);
    return (bf16 ? launch_layer_bf16 : launch_layer_f16)(ctx, a, gated, gradient, grid, stream);
}

// dX of fp32 rows: the rows dz times the transposed matrices' planes, by the layer's kernel without anything behind the product.
int32_t rows_gradient_f32(rtma_ctx* ctx, const Plan& p, const rtma_layer_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* dz, int64_t ldz, void* dX, int64_t lddx,
                          cudaStream_t stream) {
    rtma_layer_desc t{};
    t.dtype = RTMA_F32; t.d_in = p.halves * p.up; t.d_out = d->d_in; t.act = RTMA_ACT_NONE;
    t.w_stride = d->w_stride;
    Plan q{};
    q.f32 = true;
    q.halves = 1; q.up = d->d_in;
    q.ld = p.ldt;
    q.w_at = p.wt_at;
    q.tiles = p.tiles;
    cut_tiles(ctx, q.ld, 32, q.tiles, q.n_tiles, q.half, q.places);
    LayerArgs a = layer_args(ctx, q, &t, n, G, offsets, dz, ldz, nullptr, t.w_stride, nullptr, nullptr, nullptr, 0, dX, lddx, d->d_in);
    a.vo = a.go >= 16 && make_store_map(&a.map_o, RTMA_F32, dX, n, d->d_in, lddx);
    return launch_layer_f32(ctx, a, false, false, KC_GEMM_DGRAD, 2u * q.places * q.n_tiles, stream);
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
    if (X == Y || Y == W || Y == b) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: the result must not overlap the rows, the matrices or the bias", who);
    // (rows of one that are other rows of the other would be read ahead, or after they have been written)
    if (residual == Y && ldr != ldy && n > 1) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: a result in the residual branch's place must not overlap other rows of it", who);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    int64_t w_stride = d->w_stride;
    const Plan p = make_plan(ctx, d, n, G, X, ldx, W, residual, ldr, false);
    RTMA_TRY(prepare_row_call(ctx, p.end, stream));
    if (p.f32)
        RTMA_TRY(split_matrices(ctx, static_cast<const float*>(W), w_stride, w_stride ? G : 1, d->d_in, d->d_out, p.halves, p.up, ctx->arena + p.w_at, p.ld, nullptr, 0, stream));
    RTMA_TRY(lay_out_rows(ctx, p, d, n, G, X, ldx, residual, ldr, W, w_stride, stream));
    LayerArgs a = layer_args(ctx, p, d, n, G, offsets, X, ldx, W, w_stride, b, slope, residual, ldr, Y, ldy, d->d_out);
    return launch_layer(ctx, a, p, d, false, d->d_out, stream);
}

extern "C" int32_t rtma_grouped_layer_grad(rtma_ctx* ctx, const rtma_layer_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx, const void* W,
                                           const void* b, const float* slope, const void* dY, int64_t lddy, void* dZ, int64_t lddz, void* dX, int64_t lddx, void* dW,
                                           int64_t dw_stride, void* db, int64_t db_stride, float* dslope, int64_t dslope_stride, void* stream_) {
    const char* who = "rtma_grouped_layer_grad";
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_layer(ctx, who, d, n, G, offsets, slope));
    const bool gated = d->gated != 0, plain = !gated && d->act == RTMA_ACT_NONE, f32 = d->dtype == RTMA_F32;  // plain: dZ is dY
    const int halves = gated ? 2 : 1, width = plain && f32 ? d->d_out : columns_of(d), wide = halves * width;  // of dZ
    if (n > 0 && (!X || !W || !dY || (!plain && !dZ))) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: null pointer", who);
    if (db && !dW) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: the bias gradient comes with the weights'", who);
    if (dslope && d->act != RTMA_ACT_PRELU) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: a slope's gradient without PReLU", who);
    if (d->grad_dtype != d->dtype && d->grad_dtype != RTMA_F32) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: gradients of the parameters in type %d", who, d->grad_dtype);
    if (ldx < d->d_in || lddy < d->d_out || (!plain && lddz < wide) || (dX && lddx < d->d_in))
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: rows of %d and %d values lie closer than that", who, d->d_in, plain ? d->d_out : wide);
    if (!plain && n > 0) {
        if (dZ == X || dZ == dX || (dZ == dY && (gated || lddz != lddy || width != d->d_out))) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: dZ must not overlap other rows", who);
        if (row_granule(dZ, lddz, row_type_bytes(d->dtype)) < 16) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: rows of dZ off 16-byte boundaries", who);
    }
    if (n > 0 && dX && (dX == X || (dX == dY && plain))) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: dX must not overlap rows that are still read", who);
    const void* const results[] = {plain || n == 0 ? nullptr : dZ, n == 0 ? nullptr : dX, dW, db, dslope};
    for (int i = 0; i < 5; ++i) {
        if (!results[i]) continue;
        if (i < 2 && (results[i] == W || results[i] == b)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: rows of a result must not overlap the matrices or the bias", who);
        for (int j = 0; j < i; ++j)
            if (results[i] == results[j]) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: results must not overlap one another", who);
    }
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    int64_t w_stride = d->w_stride;
    const void* dz = plain ? dY : dZ;
    int64_t ldz = plain ? lddy : lddz;
    // All scratch at once: inside a capture nothing is enqueued unless everything fits.
    const Plan p = make_plan(ctx, d, n, G, X, ldx, W, dY, lddy, true);
    const bool column_sums = db && !f32 && !plain && n > 0;  // the bias gradient comes with dZ
    const Turns turns = Turns::of_pairs(gated, true, p.half);
    const size_t slot_rows = 8 * (size_t)(p.places + G), column_bytes = column_sums ? ArenaCursor::granule(sizeof(float) * slot_rows * turns.groups * wide) : 0,
                 slot_bytes = column_bytes + (dslope ? sizeof(float) * slot_rows * 4 * p.n_tiles : 0);
    size_t dw_bytes = 0;
    auto weights = [&](size_t* scratch) {
        return layer_dw(ctx, who, d, n, G, offsets, X, ldx, dz, ldz, width, dW, dw_stride, db, db_stride, !column_sums, p.end, scratch, stream);
    };
    if (dW) RTMA_TRY(weights(&dw_bytes));
    RTMA_TRY(prepare_row_call(ctx, std::max(p.end + slot_bytes, dw_bytes), stream));
    if (n > 0) {
        if (f32 && (dX || !plain))
            RTMA_TRY(split_matrices(ctx, static_cast<const float*>(W), w_stride, w_stride ? G : 1, d->d_in, d->d_out, p.halves, p.up, plain ? nullptr : ctx->arena + p.w_at, p.ld,
                                    dX ? ctx->arena + p.wt_at : nullptr, p.ldt, stream));
        RTMA_TRY(lay_out_rows(ctx, p, d, n, G, X, ldx, dY, lddy, W, w_stride, stream));
        if (plain) {
            dz = dY;
            ldz = lddy;
        } else {
            LayerArgs a = layer_args(ctx, p, d, n, G, offsets, X, ldx, W, w_stride, b, slope, dY, lddy, dZ, lddz, width);
            a.column_slots = column_sums ? reinterpret_cast<float*>(ctx->arena + p.end) : nullptr;
            a.columns = wide;
            a.slots_up = (int64_t)slot_rows;
            a.slope_slots = dslope ? reinterpret_cast<float*>(ctx->arena + p.end + column_bytes) : nullptr;
            RTMA_TRY(launch_layer(ctx, a, p, d, true, wide, stream));
        }
    }
    if (column_sums || dslope) {
        SumsArgs m{};
        m.offsets = offsets; m.n = n; m.tile_rows = PAIR_ROWS; m.tiles = p.tiles;
        m.G = G; m.places = p.places; m.n_tiles = p.n_tiles; m.columns = column_sums ? wide : 0;
        m.groups_log = turns.groups == 4 ? 2 : turns.groups - 1; m.slots_up = (int64_t)slot_rows;
        m.width = width; m.real_width = d->d_out;
        m.column_slots = reinterpret_cast<const float*>(ctx->arena + p.end); m.slope_slots = reinterpret_cast<const float*>(ctx->arena + p.end + column_bytes);
        m.db = db; m.dslope = dslope; m.db_stride = db_stride; m.dslope_stride = dslope_stride;
        m.shared = G > 1 && db_stride == 0; m.slope_shared = G > 1 && dslope_stride == 0;
        void (*kernel)(SumsArgs) = d->grad_dtype == RTMA_F32 ? layer_sums_kernel<float> : d->dtype == RTMA_BF16 ? layer_sums_kernel<__nv_bfloat16> : layer_sums_kernel<__half>;
        KernelScope ks(ctx, KC_REDUCE_SGD, stream);
        launch_kernel(kernel, dim3((unsigned)(ceil_div(m.columns, 32) + (dslope ? 1 : 0)), (unsigned)G), SUMS_THREADS, 0, stream, m);
        RTMA_LAUNCH_CHECK(ctx);
    }
    if (dX && n > 0)
        RTMA_TRY(f32 ? rows_gradient_f32(ctx, p, d, n, G, offsets, dz, ldz, dX, lddx, stream)
                     : rtma_grouped_linear_dx(ctx, d->dtype, n, G, offsets, d->d_in, p.halves * p.up, dz, ldz, W, w_stride, dX, lddx, stream));
    return dW ? weights(nullptr) : RTMA_OK;
}
