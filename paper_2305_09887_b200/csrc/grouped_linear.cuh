// What the kernels of the grouped products share: their arguments, a block's walk over its tiles, and the way of the results out.
#pragma once

#include <type_traits>

#include "rows.cuh"
#include "tc_common.cuh"

namespace grouped {

enum Mode { FORWARD, INPUT_GRADIENT, WEIGHT_GRADIENT };
constexpr int MAX_STAGES = 6;
constexpr int SMEM_MOST = 232448;  // bytes a block can have

struct LinearArgs {
    const int64_t* offsets;
    int64_t n;
    int G, span;
    int64_t tile_rows, tiles;  // rows of a row tile (forward, dx: 128; dw: at least, see fit_chunk), row tiles at most
    int m_tiles, n_tiles;      // tiles of one row tile: m_tiles (dw) x n_tiles
    int BN;
    int d_in, d_out;
    const void *A, *B;         // rows; matrices (forward, dx) or rows (dw)
    int64_t lda, ldb, w_stride;
    int va, vb;                // granules of the rows (bytes)
    int go;                    // granule of the result's rows
    int in_bulk;               // operands that bulk-tensor loads fetch: 1 the left one, 2 the right one
    bool vo;                   // the result can leave by bulk-tensor stores: map_o holds
    const void* bias;
    int64_t bias_stride;
    bool bias_overlaps;        // of two parts: an address then does not say which columns lie there
    int bias_rows;             // dw: partial sums of the bias gradient in a slot, one row per warp that adds them up
    void* out;                 // dw: the slots, [row tile][d_in + bias_rows][ldo]
    int64_t ldo;
    float *dW, *db;
    int64_t dw_stride, db_stride;
    int32_t* chunk_rows;       // dw: where the rows of a row tile are left for the reduction
    int* error_word;
    CUtensorMap map_a, map_b;  // operands that are fetched by bulk-tensor loads
    CUtensorMap map_o;         // the result (dw: the slots, one below the other)
};

#ifdef __CUDACC__
// Rows in whole steps of STEP: up to 2^31 - 1 of them with a chunk added do not fit 31 bits, their steps do.
template <int STEP>
__host__ __device__ __forceinline__ int steps_of(int rows) { return (int)(((uint32_t)rows + (STEP - 1)) / STEP); }
// The smallest chunk, of `least` steps or more, of which all parts have not more than `tiles`; by bisection.  most: steps of the largest
// part; count(c): chunks of c steps in all parts.  `tiles` is at least the number of parts.
template <class Count>
__host__ __device__ __forceinline__ int fit_chunk(int least, int most, int64_t tiles, Count count) {
    int lo = least, hi = most > least ? most : least;  // hi fits: a chunk a part
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (count(mid) <= tiles) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

struct Shared {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES];
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int abort;
    int32_t warp_sums[32];
    int32_t tile_rows;
    int32_t tile_start[RTMA_MAX_GROUPS + 1], begin[RTMA_MAX_GROUPS], rows[RTMA_MAX_GROUPS];
    alignas(16) float bias[8 * 128];  // of every drain warp's columns
};

// CLUSTER: the barrier may be signalled from the pair's other block
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, Shared& sh, int* error_word) {
    for (uint32_t i = 0; i < tc::WAIT_POLLS; ++i) {
        if (CLUSTER ? tc::mbar_try_wait_cluster(bar, parity) : tc::mbar_try_wait(bar, parity)) return true;
        if ((i & 1023u) == 1023u && *reinterpret_cast<volatile int*>(&sh.abort)) break;
    }
    *reinterpret_cast<volatile int*>(&sh.abort) = 1;
    atomicExch(error_word, 1);
    return false;
}

// A role's walk over a block's tiles and their stages.  PAIR: two blocks of a cluster share tiles of 2 BM rows, of which each sees its
// own BM (the second none or fewer where the part ends).
template <int MODE, int BM, int BK, bool PAIR = false>
struct Walk {
    int tile, part, row_tile, m0, n0;  // part: set before `at`, to one that is not behind the tile's
    int64_t row0;     // first row of the tile
    int rows, k_end;  // rows of the tile; terms of the contraction
    int k0;
    __device__ __forceinline__ bool at(const LinearArgs& a, const Shared& sh) {
        const int per = a.m_tiles * a.n_tiles;
        int rest = 0;
        row_tile = tile;
        if (per > 1) {
            row_tile = tile / per;
            rest = tile - row_tile * per;
        }
        if (row_tile >= sh.tile_start[a.G]) return false;
        m0 = 0;
        if (MODE == WEIGHT_GRADIENT && a.m_tiles > 1) {
            m0 = rest / a.n_tiles;
            rest -= m0 * a.n_tiles;
            m0 *= BM;
        }
        n0 = rest * a.BN;
        while (row_tile >= sh.tile_start[part + 1]) ++part;  // tiles come in ascending order
        const int64_t inside = (int64_t)(row_tile - sh.tile_start[part]) * sh.tile_rows;
        row0 = sh.begin[part] + inside;
        rows = (int)min((int64_t)sh.rows[part] - inside, (int64_t)sh.tile_rows);
        if (PAIR) {
            row0 += BM * (blockIdx.x & 1);
            rows -= BM * (int)(blockIdx.x & 1);
        }
        k_end = MODE == FORWARD ? a.d_in : MODE == INPUT_GRADIENT ? a.d_out : rows;
        k0 = 0;
        return true;
    }
    __device__ __forceinline__ bool first(const LinearArgs& a, const Shared& sh) {
        tile = blockIdx.x >> PAIR;
        part = 0;
        return at(a, sh);
    }
    __device__ __forceinline__ bool last_stage() const { return k0 + BK >= k_end; }
    __device__ __forceinline__ bool next(const LinearArgs& a, const Shared& sh) {  // the next stage
        if (!last_stage()) {
            k0 += BK;
            return true;
        }
        tile += gridDim.x >> PAIR;
        return at(a, sh);
    }
    __device__ __forceinline__ bool next_tile(const LinearArgs& a, const Shared& sh) {
        tile += gridDim.x >> PAIR;
        return at(a, sh);
    }
};

// The parts' rows and the numbers of their tiles; every thread of the block.
template <int MODE, int THREADS, int STEP>
__device__ __forceinline__ void lay_out(const LinearArgs& a, Shared& sh) {
    for (int g = threadIdx.x; g < a.G; g += THREADS) {
        int64_t begin, end;
        part_rows(a.offsets, a.n, g, begin, end, a.span);
        sh.begin[g] = (int32_t)begin;
        sh.rows[g] = (int32_t)(end - begin);
    }
    if (MODE == WEIGHT_GRADIENT) {
        __syncthreads();
        if (threadIdx.x < 32) {
            // Chunks of which there are not more than `tiles` fill the blocks that run at a time evenly, whatever the parts' sizes.
            const int lane = threadIdx.x;
            int most = 1;
            for (int g = lane; g < a.G; g += 32) most = max(most, sh.rows[g]);
            for (int o = 16; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
            const int chunk = fit_chunk((int)a.tile_rows / STEP, steps_of<STEP>(most), a.tiles, [&](int steps) {
                int64_t count = 0;
                for (int g = lane; g < a.G; g += 32) count += (steps_of<STEP>(sh.rows[g]) + steps - 1) / steps;
                for (int o = 16; o > 0; o >>= 1) count += __shfl_xor_sync(0xffffffffu, count, o);
                return count;
            });
            // (2^31 rows are no chunk: with fewer than 256 parts there are twice as many tiles, unless rows are so wide that 2^31 of them fit no memory.)
            const int32_t rows = chunk * STEP;
            if (lane == 0) {
                sh.tile_rows = rows;
                if (blockIdx.x == 0) *a.chunk_rows = rows;
            }
        }
    } else if (threadIdx.x == 0) {
        sh.tile_rows = (int32_t)a.tile_rows;
    }
    __syncthreads();
    number_tiles(a.offsets, a.n, a.G, sh.tile_rows, a.tiles, sh.tile_start, sh.warp_sums, a.span);
}

__device__ __forceinline__ void store_16(uint32_t dst, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 load_16(uint32_t src) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(src) : "memory");
    return v;
}

__device__ __forceinline__ void add_eight(float (&sums)[8], const float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[j] += v[j];
}

// A drain warp's results on their way out: 64 bytes of each of its 32 rows (a row per lane) at a time go through one of its slabs,
// in the map's 64-byte swizzle, so that they leave as one bulk-tensor store; boxes that would reach rows or columns that are
// not this tile's, and rows off the 16-byte boundaries, are written by the lanes.
template <class O, int SLABS>
struct Outlet {
    static constexpr int ROW = 64;
    uint32_t slabs;
    int at = 0;
    __device__ __forceinline__ static int swizzle(int row) { return (row >> 1) & 3; }
    // row0, c: place in the map; rows, cols: how much is this tile's; whole: all columns of the matrix from c on are, and end on a
    // 16-byte boundary (a store's box is cut off at the edge of the matrix only in steps of 16 bytes)
    __device__ __forceinline__ void put(const LinearArgs& a, const float (&v)[32], int64_t row0, int c, int rows, int cols, bool whole, O* out, int64_t ldo, int lane) {
        constexpr int WIDE = ROW / sizeof(O), PIECE = 16 / sizeof(O);
#pragma unroll
        for (int c0 = 0; c0 < 32; c0 += WIDE) {
            if (c0 >= cols) break;
            const uint32_t slab = slabs + at * 32 * ROW;
            if (lane == 0) tc::tma_store_wait_read_but<SLABS - 1>();  // the slab's last store has read it
            __syncwarp();
#pragma unroll
            for (int q = 0; q < ROW / 16; ++q) {
                const int e = c0 + q * PIECE;
                uint4 x;
                if constexpr (sizeof(O) == 4) {
                    x = make_uint4(__float_as_uint(v[e]), __float_as_uint(v[e + 1]), __float_as_uint(v[e + 2]), __float_as_uint(v[e + 3]));
                } else {
                    const O* tag = nullptr;
                    x = make_uint4(narrow2(v[e], v[e + 1], tag), narrow2(v[e + 2], v[e + 3], tag), narrow2(v[e + 4], v[e + 5], tag), narrow2(v[e + 6], v[e + 7], tag));
                }
                store_16(slab + lane * ROW + ((q ^ swizzle(lane)) << 4), x);
            }
            const bool bulk = a.vo && rows == 32 && (cols - c0 >= WIDE || whole);
            if (bulk) tc::fence_proxy_async_smem();
            __syncwarp();
            if (bulk) {
                if (lane == 0) {
                    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                                 ::"l"(reinterpret_cast<uint64_t>(&a.map_o)), "r"(slab), "r"(c + c0), "r"((int32_t)row0)
                                 : "memory");
                }
            } else {
                // single values, eight rows (16 in fp32) under way: one at a time, this took longer than all else
                const int x = lane % WIDE;
                constexpr int TOGETHER = 8;
                for (int r0 = lane / WIDE; r0 < rows; r0 += TOGETHER * (32 / WIDE)) {
                    O y[TOGETHER];
#pragma unroll
                    for (int i = 0; i < TOGETHER; ++i) {
                        const int r = r0 + i * (32 / WIDE);
                        const uint32_t from = slab + r * ROW + (((x / PIECE) ^ swizzle(r)) << 4) + (x % PIECE) * (int)sizeof(O);
                        if constexpr (sizeof(O) == 4) {
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(y[i]) : "r"(from) : "memory");
                        } else {
                            unsigned short bits;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(bits) : "r"(from) : "memory");
                            y[i] = *reinterpret_cast<O*>(&bits);
                        }
                    }
                    O* to = out + r0 * ldo + c0 + x;
#pragma unroll
                    for (int i = 0; i < TOGETHER; ++i, to += (32 / WIDE) * ldo)
                        if (r0 + i * (32 / WIDE) < rows && c0 + x < cols) *to = y[i];
                }
            }
            if (lane == 0) tc::tma_store_commit();  // a group for every slab, empty or not
            at = at + 1 == SLABS ? 0 : at + 1;
        }
    }
    __device__ __forceinline__ void finish(int lane) const {
        if (lane == 0) tc::tma_store_wait_all();
    }
};

// The bias of a warp's columns (chunks c, c + step, ... of 32), in shared memory.
template <class T>
struct BiasHolder {
    float* at;                 // 16-byte boundary
    const T* held = nullptr;   // of which columns: a block's tiles have the same ones most of the time
    __device__ __forceinline__ void fetch(const LinearArgs& a, int part, int n0, int c, int step, int chunks, int lane) {
        const T* bias = static_cast<const T*>(a.bias) + part * a.bias_stride + n0;
        if (bias == held && !a.bias_overlaps) return;
        held = bias;
        __syncwarp();
        for (int chunk = c, i = 0; chunk < chunks; chunk += step, ++i) {
            const int col = 32 * chunk + lane;
            at[32 * i + lane] = col < a.BN && n0 + col < a.d_out ? to_f32(bias[col]) : 0.f;
        }
        __syncwarp();
    }
    __device__ __forceinline__ void add(float (&v)[32], int i) const {
        const float4* b = reinterpret_cast<const float4*>(at + 32 * i);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float4 x = b[j];
            v[4 * j] += x.x;
            v[4 * j + 1] += x.y;
            v[4 * j + 2] += x.z;
            v[4 * j + 3] += x.w;
        }
    }
};

#endif

}  // namespace grouped

// Products of fp32 rows (grouped_split.cu): widest tiles, the partial bias sums that a dw tile leaves, the scratch that the matrices'
// planes take in forward and dx, and the launch.
constexpr int SPLIT_COLUMNS = 128, SPLIT_DW_COLUMNS = 64, SPLIT_BIAS_ROWS = 8, SPLIT_BLOCKS_PER_SM = 2;
size_t split_planes_bytes(const grouped::LinearArgs& a);
int32_t launch_split(rtma_ctx* ctx, int mode, grouped::LinearArgs& a, void* planes, int cls, cudaStream_t stream);
