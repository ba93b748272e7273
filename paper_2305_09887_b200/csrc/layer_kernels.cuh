// The kernel of whole layers (layer.cu) on 16-bit rows off 16-byte boundaries, or not many of them: what the warps that drain do.
#pragma once

#include "grouped_rows.cuh"
#include "layer.cuh"

namespace {

using namespace grouped;

// 32 values of a lane's row as they are stored; those that do not exist read as zero.
template <class T>
struct Side {
    Eight<T> e[4];
    __device__ __forceinline__ void load(const T* p, int valid, int granule) {
        if (valid >= 32 && granule == 32) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint4 &x = e[2 * i].w[0], &y = e[2 * i + 1].w[0];
                asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w), "=r"(y.x), "=r"(y.y), "=r"(y.z), "=r"(y.w)
                             : "l"(p + 16 * i));
            }
        } else if (granule >= 16 && valid % 8 == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[i].w[0] = make_uint4(0u, 0u, 0u, 0u);
                if (8 * i < valid) asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(e[i].w[0].x), "=r"(e[i].w[0].y), "=r"(e[i].w[0].z), "=r"(e[i].w[0].w) : "l"(p + 8 * i));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i].load(p + 8 * i, max(0, min(8, valid - 8 * i)), granule);
        }
    }
};

// A block's walk over its tiles, by the warps that drain: no divisions, which for every warp and tile cost as much as the results.
template <class F>
struct TileAt {
    int row_tile, rest, part, n0, rows;
    int64_t row0;
    __device__ __forceinline__ int tile(const LayerArgs& a) const { return row_tile * a.n_tiles + rest; }
    __device__ __forceinline__ bool at(const LayerArgs& a, const Shared& sh) {
        if (row_tile >= sh.tile_start[a.G]) return false;
        while (row_tile >= sh.tile_start[part + 1]) ++part;  // tiles come in ascending order
        n0 = rest * a.BN;
        const int64_t inside = (int64_t)(row_tile - sh.tile_start[part]) * (BM);
        row0 = sh.begin[part] + inside;
        rows = (int)min(sh.rows[part] - inside, (int64_t)BM);
        return true;
    }
    __device__ __forceinline__ bool first(const LayerArgs& a, const Shared& sh) {
        row_tile = blockIdx.x / a.n_tiles;
        rest = blockIdx.x - row_tile * a.n_tiles;
        part = 0;
        return at(a, sh);
    }
    __device__ __forceinline__ bool next_tile(const LayerArgs& a, const Shared& sh) {
        row_tile += a.step_rows;
        rest += a.step_rest;
        if (rest >= a.n_tiles) {
            rest -= a.n_tiles;
            ++row_tile;
        }
        return at(a, sh);
    }
};

// What a drain warp does: its rows (a quarter of the tile's) of every SLICES-th 32 columns.  The rows read beside the accumulators are
// requested 32 columns ahead, from the next tile where these are a tile's last.
template <class F, bool GRADIENT>
__device__ __forceinline__ void drain_layer(const LayerArgs& a, Shared& sh, uint32_t slabs) {
    typedef typename F::T T;
    typedef Outlet<T, F::OUT_SLABS> Out;
    constexpr bool GATED = F::GATED;
    const int act = a.act;
    const bool beside = GRADIENT || a.side;
    constexpr int SLICES = F::DRAIN_WARPS / 4, PIECE = 16 / (int)sizeof(T);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3, slice = warp >> 2;
    Out outlet{slabs + warp * F::OUT_BYTES};
    LayerBias bias{sh.bias + 1024 / F::DRAIN_WARPS * warp};
    const uint32_t tmem = sh.tmem_base + ((uint32_t)(32 * quarter) << 16);
    const int chunks = (a.BN + 31) / 32, mine = (chunks - slice + SLICES - 1) / SLICES;
    int slope_part = -1;
    float slope = 0.f;
    TileAt<F> w, ahead;
    tc::RingAt acc;
    bool more = w.first(a, sh), ahead_more = more && beside && mine > 0;
    ahead = w;
    int ahead_chunk = slice;
    Side<T> next;
    auto request = [&]() {
        if (!ahead_more) return;
        const int c = ahead.n0 + 32 * ahead_chunk, cols = min(min(32, a.BN - 32 * ahead_chunk), a.width - c);
        next.load(static_cast<const T*>(a.side) + (ahead.row0 + 32 * quarter + lane) * a.lds + c, 32 * quarter + lane < ahead.rows ? max(0, cols) : 0, a.gs);
        ahead_chunk += SLICES;
        if (ahead_chunk >= chunks) {
            ahead_chunk = slice;
            ahead_more = ahead.next_tile(a, sh);
        }
    };
    request();
    for (; more; more = w.next_tile(a, sh)) {
        const int rows = min(32, w.rows - 32 * quarter);
        const int64_t row0 = w.row0 + 32 * quarter;
        auto column = [&](int chunk) { return w.n0 + 32 * chunk; };
        auto columns = [&](int chunk) { return min(min(32, a.BN - 32 * chunk), a.width - column(chunk)); };
        if constexpr (GATED)
            bias.fetch(a, w.part, w.n0, 2 * mine, lane, static_cast<const T*>(nullptr),
                       [&](int i) { return column(slice + SLICES * (i >> 1)) + (i & 1 ? a.width : 0); }, [&](int i) { return columns(slice + SLICES * (i >> 1)); });
        else
            bias.fetch(a, w.part, w.n0, mine, lane, static_cast<const T*>(nullptr), [&](int i) { return column(slice + SLICES * i); },
                       [&](int i) { return columns(slice + SLICES * i); });
        if (act == RTMA_ACT_PRELU && w.part != slope_part) {
            slope_part = w.part;
            slope = __ldg(a.slope + w.part * a.slope_stride);
        }
        float slope_sum = 0.f;
        if (!wait_for(&sh.acc_full[acc.s], acc.phase, sh, a.error_word)) return;
        __syncwarp();
        tc::tc_fence_after_sync();
        for (int i = 0; i < mine; ++i) {
            const int chunk = slice + SLICES * i, c = column(chunk), cols = columns(chunk);
            const Side<T> side = next;
            request();
            if (rows <= 0 || cols <= 0) continue;
            const uint32_t from = tmem + acc.s * F::ACC_COLUMNS + 32 * chunk;
            const uint32_t slab = outlet.open(lane), other = GATED && GRADIENT ? outlet.open_second(lane) : 0;
            float ds = 0.f;
            // eight columns at a time, the next eight on their way from tensor memory
            uint32_t x[2][8], x2[2][8];
            tc::tmem_load_issue_8(from, x[0]);
            if constexpr (GATED) tc::tmem_load_issue_8(from + 128, x2[0]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                tc::tmem_load_wait_8(x[q & 1]);
                if constexpr (GATED) tc::tmem_load_wait_8(x2[q & 1]);
                if (q < 3) {
                    tc::tmem_load_issue_8(from + 8 * (q + 1), x[(q + 1) & 1]);
                    if constexpr (GATED) tc::tmem_load_issue_8(from + 128 + 8 * (q + 1), x2[(q + 1) & 1]);
                }
                f2 z[4], y[4], d[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    z[k] = pack2(__uint_as_float(x[q & 1][2 * k]), __uint_as_float(x[q & 1][2 * k + 1]));
                    if constexpr (GATED) y[k] = pack2(__uint_as_float(x2[q & 1][2 * k]), __uint_as_float(x2[q & 1][2 * k + 1]));
                }
                if (beside) pairs_of(side.e[q], d);
                ds += eight_results<GATED, GRADIENT>(act, beside, bias, (GATED ? 64 : 32) * i + 8 * q, 64 * i + 32 + 8 * q, slope, a.slope_slots != nullptr, cols - 8 * q, z, y, d);
                float v[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) unpack2(z[k], v[2 * k], v[2 * k + 1]);
                Out::piece(slab, lane, q, Out::pack_piece(v));
                if constexpr (GATED && GRADIENT) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) unpack2(y[k], v[2 * k], v[2 * k + 1]);
                    Out::piece(other, lane, q, Out::pack_piece(v));
                }
            }
            if (act == RTMA_ACT_PRELU && lane < rows) slope_sum += ds;  // (what the accumulator has for rows that are not there may be anything)
            T* const out = static_cast<T*>(a.out) + row0 * a.ldo + c;
            const bool whole = c + cols == a.width && a.width % PIECE == 0;
            if constexpr (GATED && GRADIENT) {
                outlet.close(a, slab, row0, c, rows, cols, false, out, a.ldo, lane);
                outlet.close(a, other, row0, a.width + c, rows, cols, whole, out + a.width, a.ldo, lane, a.width % PIECE == 0);
            } else {
                outlet.close(a, slab, row0, c, rows, cols, whole, out, a.ldo, lane);
            }
        }
        tc::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&sh.acc_empty[acc.s]);
        acc.advance(2);
        if (GRADIENT && act == RTMA_ACT_PRELU && a.slope_slots) {
            for (int o = 16; o > 0; o >>= 1) slope_sum += __shfl_xor_sync(0xffffffffu, slope_sum, o);
            if (lane == 0) a.slope_slots[(int64_t)w.tile(a) * a.slope_warps + warp] = slope_sum;
        }
    }
    outlet.finish(lane);
}

template <class T, bool GATED, bool GRADIENT>
__global__ void __launch_bounds__(Form<T, FORWARD, COPIES, GATED>::THREADS, 1) layer_copies_kernel(const __grid_constant__ LayerArgs a) {
    typedef Form<T, FORWARD, COPIES, GATED> F;
    __shared__ Shared sh;
    linear_body<F>(a, sh, [&](uint32_t slabs) { drain_layer<F, GRADIENT>(a, sh, slabs); });
}

template <class T, bool GATED, bool GRADIENT>
int32_t launch_copies_form(rtma_ctx* ctx, LayerArgs& a, unsigned grid, bool& configured, cudaStream_t stream) {
    typedef Form<T, FORWARD, COPIES, GATED> F;
    void (*kernel)(LayerArgs) = layer_copies_kernel<T, GATED, GRADIENT>;
    if (!configured) {
        RTMA_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, F::DYNAMIC_BYTES));
        configured = true;
    }
    a.step_rows = (int)grid / a.n_tiles;
    a.step_rest = (int)grid % a.n_tiles;
    launch_kernel(kernel, grid, F::THREADS, F::DYNAMIC_BYTES, stream, a);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

template <class T>
int32_t launch_copies(rtma_ctx* ctx, LayerArgs& a, bool gated, bool gradient, unsigned grid, cudaStream_t stream) {
    bool* once = ctx->layer_configured + 16 + (std::is_same<T, __half>::value ? 4 : 0);
    if (gated) return gradient ? launch_copies_form<T, true, true>(ctx, a, grid, once[3], stream) : launch_copies_form<T, true, false>(ctx, a, grid, once[2], stream);
    return gradient ? launch_copies_form<T, false, true>(ctx, a, grid, once[1], stream) : launch_copies_form<T, false, false>(ctx, a, grid, once[0], stream);
}

}  // namespace
