// What the kernels of whole layers share: products of rows whose results go through an activation, a gate or a residual branch on
// their way out (layer.cu: layer_pairs.cuh and layer_f32.cu; layer_wgrad.cu takes parts of them).
#pragma once

#include "activation.cuh"
#include "grouped_linear.cuh"

namespace grouped {

struct LayerArgs : LinearArgs {
    int width;            // columns of the result (of each of a gated layer's two matrices)
    int up;               // columns from one of the two matrices to the other
    int act;
    const float* slope;
    int64_t slope_stride;
    const void* side;     // rows read on the way out: the residual branch (or none), or the result's gradient
    int64_t lds;
    float* slope_slots;   // gradient, PReLU: what the warps that drain have of the slope's gradient, [place + part][block of the pair,
                          // quarter of its rows][tile of columns][slice]
    int half;             // columns that each block of a pair brings of the matrix (gated: of one of the two)
    int places;           // pairs that share a tile's columns
    int bias_up, bias_width;  // as width and the distance of the two matrices, in the bias (width may be rounded up)
    CUtensorMap map_side;
    float* column_slots;  // gradient: sums of dZ's columns, [group of warps (Turns)][8 (places + parts)][columns]
    int64_t slots_up;     // from one group's slots to the next's, in rows
    int columns;
};

#ifdef __CUDACC__
constexpr int PAIR_BM = 128;            // rows of a tile that a block of a pair has
constexpr int SLAB_BYTES = 32 * 128;    // of an operand: 32 rows of 64 16-bit values
// A pair's walk down its row tiles; rows and row0 are the block's own.
struct PairWalk {
    int t, end, part, left;  // left: rows of the part from the tile's first on
    int64_t first_row;
    __device__ __forceinline__ bool open(const LayerArgs& a, const Shared& sh) {
        const int64_t tiles = sh.tile_start[a.G];
        const int place = (blockIdx.x >> 1) / a.n_tiles;
        t = (int)(tiles * place / a.places);
        end = (int)(tiles * (place + 1) / a.places);
        if (t >= end) return false;
        part = part_of_tile(sh.tile_start, a.G, t);
        return at(sh);
    }
    __device__ __forceinline__ bool at(const Shared& sh) {
        const int inside = (t - sh.tile_start[part]) * 2 * PAIR_BM;
        first_row = (int64_t)sh.begin[part] + inside;
        left = sh.rows[part] - inside;
        return true;
    }
    __device__ __forceinline__ bool next(const Shared& sh) {
        if (++t >= end) return false;
        if (t >= sh.tile_start[part + 1]) {
            do ++part;
            while (t >= sh.tile_start[part + 1]);
            return at(sh);
        }
        first_row += 2 * PAIR_BM;
        left -= 2 * PAIR_BM;
        return true;
    }
    __device__ __forceinline__ bool part_ends(const Shared& sh) const { return t + 1 >= end || t + 1 >= sh.tile_start[part + 1]; }
};

// The bias of a warp's columns in shared memory: 32 at a time, `chunks` of them.  Held for as long as part and column stay.
struct LayerBias {
    float* at;  // 16-byte boundary
    int part = -1, n0 = -1;
    // column(i): where chunk i starts in the bias; edge(i): how many columns of it there are
    template <class T, class Column, class Edge>
    __device__ __forceinline__ void fetch(const LayerArgs& a, int of_part, int of_n0, int chunks, int lane, const T*, Column column, Edge edge) {
        if (of_part == part && of_n0 == n0) return;
        part = of_part;
        n0 = of_n0;
        const T* bias = static_cast<const T*>(a.bias) + part * a.bias_stride;  // (none: zeros)
        __syncwarp();
        for (int i = 0; i < chunks; ++i) at[32 * i + lane] = a.bias && lane < edge(i) ? to_f32(bias[column(i) + lane]) : 0.f;
        __syncwarp();
    }
    // eight of them, from the one numbered j on, added to v
    __device__ __forceinline__ void add(f2 (&v)[4], int j) const {
        const float4* b = reinterpret_cast<const float4*>(at + j);
        const float4 x = b[0], y = b[1];
        v[0] = add2(v[0], pack2(x.x, x.y));
        v[1] = add2(v[1], pack2(x.z, x.w));
        v[2] = add2(v[2], pack2(y.x, y.y));
        v[3] = add2(v[3], pack2(y.z, y.w));
    }
};

// Narrow tiles: where columns leave warps without any, groups of warps take tiles by turns, out of four accumulators instead of two (fp16 300,000 x 100 ->
// 47, first step of the gradient 46 -> 41 us; fp32 700,000 x 64 -> 2 125 -> 99, 64 -> 64 135 -> 105).
struct Turns {
    int groups, slices, buffers, spacing;  // slices: warps for each quarter of the rows that share a tile's columns
    // wide: columns of a tile, of which a warp takes 32 (or every fourth 32) of its rows (fp32: half of the columns, as a warp takes 64)
    __host__ __device__ explicit Turns(int wide) {
        slices = wide <= 32 ? 1 : wide <= 64 ? 2 : 4;
        groups = 4 / slices;
        buffers = groups > 1 ? 4 : 2;
        spacing = 512 / buffers;
    }
    // 16-bit rows.  Not for the gradient of gated layers: the registers that it takes cost 500,000 x 256 -> 2 x 512 387 -> 412 us
    // without any turn taken
    __host__ __device__ static Turns of_pairs(bool gated, bool gradient, int half) { return Turns(gated ? (gradient ? 256 : half) : 2 * half); }
};

// Values from `valid` on become zero: tensor memory may hold anything in columns that are not the tile's, and a sum must not see it.
__device__ __forceinline__ void cut_eight(f2 (&x)[4], int valid) {
    if (valid >= 8) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        unpack2(x[i], a, b);
        x[i] = pack2(2 * i < valid ? a : 0.f, 2 * i + 1 < valid ? b : 0.f);
    }
}

// Eight of a lane's results.  z (and y, a gated layer's second factors): sums of the products, bias j.. added here; d: the row that is read
// beside them (beside).  summed: the slope's gradient is wanted.  z (and y) become what is stored; returns the slope's gradient.  valid: how many are the tile's.
template <bool GATED, bool GRADIENT>
__device__ __forceinline__ float eight_results(int act, bool beside, const LayerBias& bias, int j, int j2, float slope, bool summed, int valid, f2 (&z)[4], f2 (&y)[4], const f2 (&d)[4]) {
    float ds = 0.f;
    bias.add(z, j);
    if constexpr (GATED) bias.add(y, j2);
    if constexpr (GRADIENT) {
        if (act == RTMA_ACT_PRELU && summed) {
            cut_eight(z, valid);
            if constexpr (GATED) cut_eight(y, valid);
        }
        if constexpr (GATED) {
            f2 dz[4], dy[4];
            ds = gate_back(act, slope, z, y, d, dz, dy);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[i] = dz[i];
                y[i] = dy[i];
            }
        } else {
            f2 dz[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) dz[i] = d[i];
            ds = activate_back(act, slope, z, dz);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = dz[i];
        }
    } else {
        activate(act, slope, z);
        if constexpr (GATED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = beside ? fma2(z[i], y[i], d[i]) : mul2(z[i], y[i]);
        } else if (beside) {
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = add2(z[i], d[i]);
        }
    }
    return ds;
}
// f of the activation (and of whether rows are read beside the sums) as constants
template <bool GRADIENT, class Call>
__device__ __forceinline__ void with_activation(const LayerArgs& a, Call f) {
    auto beside = [&](auto ACT) {
        if (GRADIENT || a.side) f(ACT, std::true_type());
        else f(ACT, std::false_type());
    };
    switch (a.act) {
        case RTMA_ACT_NONE: beside(std::integral_constant<int, RTMA_ACT_NONE>()); break;
        case RTMA_ACT_RELU: beside(std::integral_constant<int, RTMA_ACT_RELU>()); break;
        case RTMA_ACT_PRELU: beside(std::integral_constant<int, RTMA_ACT_PRELU>()); break;
        default: beside(std::integral_constant<int, RTMA_ACT_SILU>()); break;
    }
}
#endif

}  // namespace grouped

// fp32 rows on 16-byte boundaries (layer_f32.cu).  a.B: planes that the matrices have been split into, of a.ldb columns.
int32_t launch_layer_f32(rtma_ctx* ctx, grouped::LayerArgs& a, bool gated, bool gradient, int cls, unsigned grid, cudaStream_t stream);
// The matrices [part][d_in][halves * width] as planes [part][3][d_in][ld], the halves by turns of 32 columns, and (transposed not NULL) as planes
// [part][3][halves * up][ldt] of their transposes, zeros for what `up` has above width.
int32_t split_matrices(rtma_ctx* ctx, const float* W, int64_t w_stride, int parts, int d_in, int width, int halves, int up, void* planes, int ld, void* transposed, int ldt,
                       cudaStream_t stream);
// 16-bit rows on 16-byte boundaries (layer_pairs.cuh).
int32_t launch_layer_bf16(rtma_ctx* ctx, grouped::LayerArgs& a, bool gated, bool gradient, unsigned grid, cudaStream_t stream);
int32_t launch_layer_f16(rtma_ctx* ctx, grouped::LayerArgs& a, bool gated, bool gradient, unsigned grid, cudaStream_t stream);
// The weight gradient of rows on 16-byte boundaries (layer_wgrad.cu), from dZ with halves of `width` columns; in the scratch from `at` on.  sums: db is formed
// here.  scratch: only says how much of it the call takes, from its start.
int32_t layer_dw(rtma_ctx* ctx, const char* who, const rtma_layer_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx, const void* dZ,
                 int64_t lddz, int width, void* dW, int64_t dw_stride, void* db, int64_t db_stride, bool sums, size_t at, size_t* scratch, cudaStream_t stream);
