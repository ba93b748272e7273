// The weight gradient of a layer (layer.cu) from rows on 16-byte boundaries: dW_g = X_g^T dZ_g, db_g = the column sums of dZ_g.
//
// Pairs of blocks (MMAs of 256 x up to 256 over 64 rows a stage); rows run across both operands, so that both come as they lie.  The
// left operand (256 columns a tile) is X or dZ, whichever makes fewer MMAs; every stage's 32 KB a block come from the L2 cache, which is what
// bounds it: 500,000 x 256 x 1,024 in bf16 278 us (0.94 PFLOP/s; 7.4 TB/s from that cache), 500,000 x 256 x 256 106 us (4.8 TB/s from memory);
// as tiles of 128 x 128 in grouped_linear.cu 456 and 127.  The parts' rows are cut into chunks as there, one slot of fp32 sums for each, added up by a second kernel.
//
// The tensor cores truncate when they accumulate: sixteen warps take the accumulator after every 128 rows and add it up in registers, rounded to
// nearest, a quarter of a row's columns in a lane.  The same warps take dZ's column sums from the stages where no kernel before has (layers without activation
// or gate: 500,000 x 256 x 1,024 351 us; as products with ones by mma.sync, which the MMAs wait for, 415).
#include <algorithm>

#include "layer.cuh"
#include "split.cuh"

RTMA_BOUNDS_TU()

namespace {

using namespace grouped;

constexpr int LEFT = 256, BK = 64, STAGES = 6, STAGE_BYTES = 2 * 128 * 128, DRAIN_WARPS = 16, THREADS = 32 * (DRAIN_WARPS + 4);
constexpr int DYNAMIC_BYTES = 1024 + STAGES * STAGE_BYTES;
constexpr int ACC_STAGES = 2;  // of 64 rows, after which the accumulator is taken
constexpr int DW_WAVES = 2;    // tiles for every pair that runs at a time
// fp32 rows: 32 of them a stage, 64 columns of the right operand in a block
constexpr int F32_BK = 32, F32_HALF = 64, RAW_STAGES = 3, RAW_BYTES = F32_BK * (128 + F32_HALF) * 4, F32_STAGES = 3, ATOM_BYTES = 3 * F32_BK * 64 * 2;
constexpr int F32_DRAIN_WARPS = 8, SPLIT_WARPS = 12, F32_THREADS = 32 * (F32_DRAIN_WARPS + 4 + SPLIT_WARPS);
constexpr int F32_DYNAMIC_BYTES = 1024 + RAW_STAGES * RAW_BYTES + F32_STAGES * 3 * ATOM_BYTES;
constexpr int F32_OTHER_REGISTERS = 64;  // 256 x 104 + 512 x 64 = 59,392 of 768 x 80
constexpr int SUMS_REGISTERS = 104, OTHER_REGISTERS = 64;  // 512 x 104 + 128 x 64 = 640 x 96

struct GradArgs : LinearArgs {  // A, map_a: the left operand, B, map_b: the right one
    int left, right;   // their widths
    bool swapped;      // dZ is the left one
    int left_half, half;  // columns that a block brings, of the left one 64 or 128
    bool sums;         // of dZ's columns are wanted
    int sum_rows;      // sums of dZ's columns in a slot, behind the weights: of as many shares of the rows
    float* slots;      // [row tile][d_in + sum_rows][ldo]
    int width, real_width;  // of dZ's halves, with and without what was rounded up
    int real_out;      // columns of dW
    void *to_w, *to_b; // dW and db, in float or in the rows' type
    int first_row, rows;  // of the slots, which a reduction adds up: d_in of dW, then db
    bool all_parts;       // over all parts
};

template <int SIZE>
__device__ __forceinline__ void copy(uint32_t dst, const void* src, int bytes) {  // the rest of the SIZE bytes becomes zero
    asm volatile("cp.async.cg.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(bytes), "n"(SIZE) : "memory");
}

struct GradShared : Shared {
    uint64_t ready[STAGES], free[STAGES];  // stages that have come, in either block; whose columns have been summed
};

template <int STEP>
struct GradWalk {
    int tile, row_tile, part, m0, n0, k_end, k0;
    int64_t row0;
    __device__ __forceinline__ bool at(const GradArgs& a, const Shared& sh) {
        const int per = a.m_tiles * a.n_tiles;
        row_tile = tile / per;
        if (row_tile >= sh.tile_start[a.G]) return false;
        const int rest = tile - row_tile * per;
        m0 = rest / a.n_tiles;
        n0 = (rest - m0 * a.n_tiles) * 2 * a.half;
        m0 *= 2 * a.left_half;
        while (row_tile >= sh.tile_start[part + 1]) ++part;  // tiles come in ascending order
        const int64_t inside = (int64_t)(row_tile - sh.tile_start[part]) * sh.tile_rows;
        row0 = sh.begin[part] + inside;
        k_end = (int)min((int64_t)sh.rows[part] - inside, (int64_t)sh.tile_rows);
        k0 = 0;
        return true;
    }
    __device__ __forceinline__ bool first(const GradArgs& a, const Shared& sh) {
        tile = blockIdx.x >> 1;
        part = 0;
        return at(a, sh);
    }
    __device__ __forceinline__ bool next_tile(const GradArgs& a, const Shared& sh) {
        tile += gridDim.x >> 1;
        return at(a, sh);
    }
    __device__ __forceinline__ bool last_stage() const { return k0 + STEP >= k_end; }
    __device__ __forceinline__ bool next(const GradArgs& a, const Shared& sh) {  // the next stage
        if (!last_stage()) {
            k0 += STEP;
            return true;
        }
        return next_tile(a, sh);
    }
    // whether this tile's block sums columns of dZ: once for each, in the first tile of X's columns
    __device__ __forceinline__ bool sums(const GradArgs& a) const { return a.sums && (a.swapped ? n0 : m0) == 0; }
};

// A warp for either operand (500,000 x 256 x 1,024: one for both 286 us, these two 278).  Rows behind the end of a chunk belong to
// another part: the last stage's rows are copied by the lanes, with zeros behind them.
template <class T, bool RIGHT>
__device__ __forceinline__ void grad_producer(const GradArgs& a, GradShared& sh, uint8_t* ring, int rank, int lane) {
    const CUtensorMap* const map = RIGHT ? &a.map_b : &a.map_a;
    if (lane == 0) tc::prefetch_tensormap(map);
    const int atoms = RIGHT ? (a.half + 63) / 64 : a.left_half / 64, up = (RIGHT ? a.half : a.left_half) * rank, width = RIGHT ? a.right : a.left;
    ring += RIGHT ? 4 * SLAB_BYTES : 0;
    GradWalk<BK> w;
    tc::RingAt at;
    int filled = 0;  // stages, STAGES at most
    bool ok = true;
    for (bool more = w.first(a, sh); more; more = w.next(a, sh), at.advance(STAGES)) {
        if (!wait_for<true>(&sh.empty[at.s], at.phase ^ 1u, sh, a.error_word) || (a.sums && !wait_for(&sh.free[at.s], at.phase ^ 1u, sh, a.error_word))) {
            ok = false;
            break;
        }
        filled = min(filled + 1, STAGES);
        uint8_t* stage = ring + at.s * STAGE_BYTES;
        const uint32_t bar = tc::leader_addr(&sh.full[at.s]);
        const int first = (RIGHT ? w.n0 : w.m0) + up;
        if (w.k0 + BK > w.k_end) {
            const int64_t ld = RIGHT ? a.ldb : a.lda;
            const T* const from = static_cast<const T*>(RIGHT ? a.B : a.A);
            for (int j = lane; j < atoms * 512; j += 32) {
                const int atom = j >> 9, row = j >> 3 & 63, unit = j & 7, k = w.k0 + row, c = first + 64 * atom + 8 * unit;
                const int valid = k < w.k_end ? max(0, min(8, width - c)) : 0;
                copy<16>(tc::smem_u32(stage) + atom * 2 * SLAB_BYTES + row * 128 + ((unit ^ (row & 7)) << 4), valid ? from + (w.row0 + k) * ld + c : from, valid * (int)sizeof(T));
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            tc::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive_cluster(bar);
        } else if (lane == 0) {
            if (rank == 0) tc::mbar_arrive_expect_tx(&sh.full[at.s], 2 * atoms * 2 * SLAB_BYTES);
            else tc::mbar_arrive_remote(bar);
            for (int i = 0; i < atoms; ++i) tc::tma_load_3d_pair(stage + i * 2 * SLAB_BYTES, map, bar, first + 64 * i, (int)w.row0 + w.k0, 0);
        }
        __syncwarp();
    }
    // No signal stays under way: every stage filled is waited for until both blocks have it back or, after a give-up, until its loads have
    // landed (the first block, for both).
    for (int i = 0; i < filled; ++i) {
        const int back = filled - i, s = (at.s - back + STAGES) % STAGES;
        const uint32_t parity = s < at.s ? at.phase : at.phase ^ 1u;
        if (!ok || !wait_for<true>(&sh.empty[s], parity, sh, a.error_word) || (a.sums && !wait_for(&sh.free[s], parity, sh, a.error_word))) {
            ok = false;
            if (rank == 0)
                for (uint32_t k = 0; k < (1u << 14) && !tc::mbar_try_wait_cluster(&sh.full[s], parity); ++k) {}
        }
    }
}

template <class T>
__device__ __forceinline__ void grad_multiplier(const GradArgs& a, GradShared& sh, uint32_t ring) {
    const uint32_t format = std::is_same<T, __half>::value ? 0u : 1u;  // fp16 or bf16 operands, fp32 sums
    const uint32_t idesc = (1u << 4) | (format << 7) | (format << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(2 * a.half >> 3) << 17) | ((uint32_t)(LEFT >> 4) << 24);
    const uint64_t desc = tc::smem_desc_sw128(0, 2 * SLAB_BYTES, 1024);  // atoms of 64 columns lie two slabs apart
    GradWalk<BK> w;
    tc::RingAt at, acc;
    int held = 0;  // stages in the accumulator
    for (bool more = w.first(a, sh); more; more = w.next(a, sh)) {
        if (held == 0 && !wait_for<true>(&sh.acc_empty[acc.s], acc.phase ^ 1u, sh, a.error_word)) return;
        if (!wait_for<true>(&sh.full[at.s], at.phase, sh, a.error_word)) return;
        tc::tc_fence_after_sync();
        __syncwarp();
        if (a.sums) tc::commit_pair_by_warp(&sh.ready[at.s]);  // (both blocks learn of the stage when the one before has been multiplied)
        const uint32_t d = sh.tmem_base + acc.s * 256, stage = ring + at.s * STAGE_BYTES;
        const uint64_t da = desc + (stage >> 4), db = da + (4 * SLAB_BYTES >> 4);
        const int steps = (min(BK, w.k_end - w.k0) + 15) >> 4;
#pragma unroll
        for (int k = 0; k < BK / 16; ++k)
            if (k < steps) tc::mma_pair_by_warp(d, da + 128 * k, db + 128 * k, idesc, k || held ? 1u : 0u);
        tc::commit_pair_by_warp(&sh.empty[at.s]);
        at.advance(STAGES);
        if (++held == ACC_STAGES || w.last_stage()) {
            held = 0;
            tc::commit_pair_by_warp(&sh.acc_full[acc.s]);
            acc.advance(2);
        }
    }
}

// Column sums of dZ, beside the MMAs: the drain warps take 16 columns of half of a stage's rows each.
template <class T>
struct ColumnSums {
    f2 of[2];  // of columns lane / 4 and 8 behind it, of a lane's rows: even ones, odd ones
    __device__ __forceinline__ void clear() { of[0] = of[1] = pack2(0.f, 0.f); }
    __device__ __forceinline__ void add(uint32_t columns, int which, int lane, int rows) {  // columns: of dZ in the stage; which: of the 16 warps
        const int m = which >> 1;
        // four 8 x 8 blocks of 16 x 16 values: columns .. + 7 and + 8 .. + 15 of rows .. + 7, then of rows + 8 .. + 15
        const uint32_t from = columns + (m >> 2) * 2 * SLAB_BYTES + (32 * (which & 1) + 8 * (lane >> 4) + (lane & 7)) * 128 + (((2 * (m & 3) + (lane >> 3 & 1)) ^ (lane & 7)) << 4);
        uint32_t x[2][4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                         : "=r"(x[k][0]), "=r"(x[k][1]), "=r"(x[k][2]), "=r"(x[k][3])
                         : "r"(from + 2048 * k)
                         : "memory");
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (32 * (which & 1) + 16 * k >= rows) break;  // (rows behind the last are zeros up to 64 if there are any)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float a, b;
                widen2(x[k][i], a, b, static_cast<const T*>(nullptr));
                of[i & 1] = add2(of[i & 1], pack2(a, b));
            }
        }
    }
    __device__ __forceinline__ float total(int h) const {  // of all lanes' rows
        float s = halves_sum(of[h]);
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        return s + __shfl_xor_sync(0xffffffffu, s, 2);
    }
};

// before(w, k0): what is done before the accumulator of the rows from k0 on is waited for; after(w): at the end of a tile.
// RING, SPACING: of accumulators and their columns; SLICES: of columns, a warp for each quarter of the rows.  TURNED: of every 64 columns of an operand the upper 32 lie with the halves of each eight the other way
// around (see grad_f32_splitter).
template <int STEP, int TAKEN, int RING, int SPACING, int SLICES, bool TURNED, class S, class Before, class After>
__device__ __forceinline__ void grad_drain(const GradArgs& a, S& sh, int rank, Before before, After after) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3, slice = warp >> 2;
    const int per = 2 * a.half / SLICES;  // columns of a warp: a multiple of 8, 64 at most
    const uint32_t tmem = sh.tmem_base + ((uint32_t)(32 * quarter) << 16) + per * slice;
    GradWalk<STEP> w;
    tc::RingAt acc;
    for (bool more = w.first(a, sh); more; more = w.next_tile(a, sh)) {
        f2 total[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) total[j] = pack2(0.f, 0.f);
        for (int k0 = 0; k0 < w.k_end; k0 += TAKEN) {
            if (!before(w, k0)) return;
            if (!wait_for<true>(&sh.acc_full[acc.s], acc.phase, sh, a.error_word)) return;
            __syncwarp();
            tc::tc_fence_after_sync();
            const uint32_t from = tmem + acc.s * SPACING;
            uint32_t x[2][8];
            tc::tmem_load_issue_8(from, x[0]);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                tc::tmem_load_wait_8(x[q & 1]);
                const bool last = q == 7 || 8 * (q + 1) >= per;
                if (!last) tc::tmem_load_issue_8(from + 8 * (q + 1), x[(q + 1) & 1]);
#pragma unroll
                for (int j = 0; j < 4; ++j) total[4 * q + j] = add2(total[4 * q + j], pack2(__uint_as_float(x[q & 1][2 * j]), __uint_as_float(x[q & 1][2 * j + 1])));
                if (last) break;
            }
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive_remote(tc::leader_addr(&sh.acc_empty[acc.s]));  // (a pair's warps all report to the first block)
            acc.advance(RING);
        }
        after(w);
        const int m = w.m0 + a.left_half * rank + 32 * quarter + (TURNED && (quarter & 1) ? lane ^ 4 : lane), n = w.n0 + per * slice;
        const int cols = min(per, a.right - n);
        if constexpr (TURNED) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if ((per * slice + 8 * q) % a.half < 32) continue;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const f2 t = total[4 * q + j];
                    total[4 * q + j] = total[4 * q + 2 + j];
                    total[4 * q + 2 + j] = t;
                }
            }
        }
        if (32 * quarter < a.left_half && m < a.left && cols > 0) {
            float* const slot = a.slots + (int64_t)w.row_tile * (a.d_in + a.sum_rows) * a.ldo;
            if (a.swapped) {  // a lane's column of dZ: neighbours beside one another
                float* to = slot + (int64_t)n * a.ldo + m;
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    float x, y;
                    unpack2(total[j], x, y);
                    if (2 * j < cols) to[0] = x;
                    if (2 * j + 1 < cols) to[a.ldo] = y;
                    to += 2 * a.ldo;
                }
            } else {  // a lane's row of dW (the slots' rows are padded to 32 bytes)
                float* to = slot + (int64_t)m * a.ldo + n;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) unpack2(total[4 * q + j], v[2 * j], v[2 * j + 1]);
                    if (8 * q < cols)
                        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 8 * q), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]),
                                     "f"(v[6]), "f"(v[7])
                                     : "memory");
                }
            }
        }
    }
}

template <class T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) layer_wgrad_kernel(const __grid_constant__ GradArgs a) {
    static_assert(DYNAMIC_BYTES + sizeof(GradShared) <= SMEM_MOST && STAGES <= MAX_STAGES, "shared memory of a block");
    extern __shared__ uint8_t raw[];
    __shared__ GradShared sh;
    uint8_t* const ring_bytes = raw + ((1024u - (tc::smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t ring = tc::smem_u32(ring_bytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            tc::mbar_init(&sh.full[s], 4);  // both blocks', of either operand
            tc::mbar_init(&sh.empty[s], 1);
            tc::mbar_init(&sh.ready[s], 1);
            tc::mbar_init(&sh.free[s], DRAIN_WARPS);
        }
        for (int b = 0; b < 2; ++b) {
            tc::mbar_init(&sh.acc_full[b], 1);
            tc::mbar_init(&sh.acc_empty[b], 2 * DRAIN_WARPS);
        }
        sh.abort = 0;
        tc::fence_barrier_init();
    }
    if (warp == DRAIN_WARPS) {
        tc::tmem_alloc_pair(&sh.tmem_base, 512);
        tc::tmem_relinquish_pair();
    }
    wait_for_kernel_before();
    lay_out<WEIGHT_GRADIENT, THREADS, BK>(a, sh);
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();  // both blocks' barriers and tensor memory exist before either is signalled
    tc::tc_fence_after_sync();
    const int rank = (int)tc::cluster_rank();
    if (warp < DRAIN_WARPS) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SUMS_REGISTERS));
        tc::RingAt at;
        ColumnSums<T> sums;
        sums.clear();
        grad_drain<BK, ACC_STAGES * BK, 2, 256, DRAIN_WARPS / 4, false>(
            a, sh, rank,
            [&](const GradWalk<BK>& w, int k0) {
                if (!a.sums) return true;
                for (int k = k0; k < min(k0 + ACC_STAGES * BK, w.k_end); k += BK) {
                    if (!wait_for<true>(&sh.ready[at.s], at.phase, sh, a.error_word)) return false;
                    __syncwarp();
                    if (w.sums(a)) sums.add(ring + at.s * STAGE_BYTES + (a.swapped ? 0 : 4 * SLAB_BYTES), warp, lane, w.k_end - k);
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&sh.free[at.s]);
                    at.advance(STAGES);
                }
                return true;
            },
            [&](const GradWalk<BK>& w) {
                if (!w.sums(a)) return;
                const int of_block = a.swapped ? a.left_half : a.half, first = a.swapped ? w.m0 + a.left_half * rank : w.n0 + a.half * rank;
                float* const to = a.slots + ((int64_t)w.row_tile * (a.d_in + a.sum_rows) + a.d_in + (warp & 1)) * a.ldo + first;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float s = sums.total(h);
                    const int j = 16 * (warp >> 1) + 8 * h + (lane >> 2);
                    if ((lane & 3) == 0 && j < of_block && first + j < a.d_out) to[j] = s;
                }
                sums.clear();
            });
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGISTERS));
        if (warp == DRAIN_WARPS && rank == 0) grad_multiplier<T>(a, sh, ring);
        if (warp == DRAIN_WARPS + 1) grad_producer<T, false>(a, sh, ring_bytes, rank, lane);
        if (warp == DRAIN_WARPS + 2) grad_producer<T, true>(a, sh, ring_bytes, rank, lane);
    }
    __syncwarp();
    if (*reinterpret_cast<volatile int*>(&sh.abort)) __nanosleep(1000000);  // a wait ran out: copies and MMAs under way land before the block ends
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();  // neither block leaves while the other may still signal it or read its operands
    if (warp == DRAIN_WARPS) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc_pair(sh.tmem_base, 512);
    }
}

// ---- fp32 rows ----------------------------------------------------------------------------------
// Six MMAs a product on three bf16 numbers a value, a fresh accumulator for every 32 rows (layer_f32.cu); tiles of 256 x 128.  Splitting is what bounds
// it (100,000 x 128 x 512: 94 us, 75 with nothing split; eight warps with fewer registers and tiles of twice the width 150): twelve warps do it, four for
// every 64 columns, always the same ones, so that they add up dZ's columns on the way.  40 bytes a thread are spilled, of warps that drain.
struct GradF32Shared : Shared {
    uint64_t raw_full[RAW_STAGES], raw_free[RAW_STAGES];
};

__device__ __forceinline__ void grad_f32_producer(const GradArgs& a, GradF32Shared& sh, uint8_t* raw, int rank) {
    tc::prefetch_tensormap(&a.map_a);
    tc::prefetch_tensormap(&a.map_b);
    const int left_boxes = a.left_half / 32, boxes = (a.half + 31) / 32;
    GradWalk<F32_BK> w;
    tc::RingAt at;
    for (bool more = w.first(a, sh); more; more = w.next(a, sh), at.advance(RAW_STAGES)) {
        if (!wait_for(&sh.raw_free[at.s], at.phase ^ 1u, sh, a.error_word)) return;
        uint8_t* stage = raw + at.s * RAW_BYTES;
        uint64_t* bar = &sh.raw_full[at.s];
        tc::mbar_arrive_expect_tx(bar, (left_boxes + boxes) * 4096);
        const int row = (int)w.row0 + w.k0;
        for (int i = 0; i < left_boxes; ++i) tc::tma_load_3d(stage + 4096 * i, &a.map_a, bar, 2 * (w.m0 + a.left_half * rank + 32 * i), row, 0);
        for (int i = 0; i < boxes; ++i) tc::tma_load_3d(stage + 4096 * (4 + i), &a.map_b, bar, 2 * (w.n0 + a.half * rank + 32 * i), row, 0);
    }
}

// which: 4 * atom (two of the left operand, one of the right one) + quarter of the rows.  A thread has eight columns of a row; those of an atom's upper 32
// read the halves of their eight the other way around, so that no two of eight threads are in one bank, and leave them so: the results' columns are
// put right once a tile.
__device__ __forceinline__ void grad_f32_splitter(const GradArgs& a, GradF32Shared& sh, uint32_t raw, uint32_t planes, int rank, int which, int lane) {
    const int atom = which >> 2, unit = lane & 7, turned = unit >> 2;
    const bool of_dz = (atom < 2) == a.swapped;
    GradWalk<F32_BK> w;
    tc::RingAt at, raw_at;
    int filled = 0;  // stages, F32_STAGES at most
    float sums[8], total[8];  // a lane's columns; sums of 16 stages are added to total, so that not every value meets a long sum
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[j] = total[j] = 0.f;
    for (bool more = w.first(a, sh); more; more = w.next(a, sh)) {
        if (!wait_for(&sh.raw_full[raw_at.s], raw_at.phase, sh, a.error_word)) return;
        if (!wait_for<true>(&sh.empty[at.s], at.phase ^ 1u, sh, a.error_word)) return;
        __syncwarp();
        const uint32_t from = raw + raw_at.s * RAW_BYTES + (2 * atom + turned) * 4096, to = planes + (3 * at.s + atom) * ATOM_BYTES;
        uint32_t v[2][8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = 8 * (which & 3) + 4 * i + (lane >> 3);
            const uint32_t line = from + row * 128;
            const uint4 x = load_16(line + (((2 * (unit & 3) + turned) ^ (row & 7)) << 4)), y = load_16(line + (((2 * (unit & 3) + 1 - turned) ^ (row & 7)) << 4));
            v[i][0] = x.x; v[i][1] = x.y; v[i][2] = x.z; v[i][3] = x.w;
            v[i][4] = y.x; v[i][5] = y.y; v[i][6] = y.z; v[i][7] = y.w;
        }
        if (w.k0 + F32_BK > w.k_end) {  // rows behind the chunk are another part's
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = w.k0 + 8 * (which & 3) + 4 * i + (lane >> 3) < w.k_end ? v[i][j] : 0u;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = 8 * (which & 3) + 4 * i + (lane >> 3);
            if (of_dz) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[j] += __uint_as_float(v[i][j]);
            }
            uint4 p[3];
            split_eight(v[i], p);
#pragma unroll
            for (int k = 0; k < 3; ++k) store_16(to + k * (ATOM_BYTES / 3) + row * 128 + ((unit ^ (row & 7)) << 4), p[k]);
        }
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            tc::mbar_arrive(&sh.raw_free[raw_at.s]);
            tc::mbar_arrive_written(tc::leader_addr(&sh.full[at.s]));
        }
        raw_at.advance(RAW_STAGES);
        at.advance(F32_STAGES);
        filled = min(filled + 1, F32_STAGES);
        if (of_dz && (w.last_stage() || (w.k0 / F32_BK) % 16 == 15)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                total[j] += sums[j];
                sums[j] = 0.f;
            }
        }
        if (w.last_stage() && of_dz) {
            const int left = a.swapped ? a.left_half - 64 * atom : a.half, first = a.swapped ? w.m0 + a.left_half * rank + 64 * atom : w.n0 + a.half * rank;
            float* const to_sums = a.slots + ((int64_t)w.row_tile * (a.d_in + a.sum_rows) + a.d_in + (which & 3)) * a.ldo + first;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float s = total[j] + __shfl_xor_sync(0xffffffffu, total[j], 8);
                s += __shfl_xor_sync(0xffffffffu, s, 16);
                const int c = 8 * unit + (j ^ (4 * turned));
                if (w.sums(a) && lane < 8 && c < left && first + c < a.d_out) to_sums[c] = s;
                total[j] = 0.f;
            }
        }
    }
    // No signal stays under way: the last stages are waited for.
    for (int i = 0; i < filled; ++i) {
        const int back = filled - i, s = (at.s - back + F32_STAGES) % F32_STAGES;
        if (!wait_for<true>(&sh.empty[s], s < at.s ? at.phase : at.phase ^ 1u, sh, a.error_word)) return;
    }
}

__device__ __forceinline__ void grad_f32_multiplier(const GradArgs& a, GradF32Shared& sh, uint32_t planes) {
    const uint32_t idesc = tc::idesc_bf16(LEFT, 2 * a.half, true, true);
    constexpr uint32_t plane = ATOM_BYTES / 3 >> 4;
    const uint64_t desc = tc::smem_desc_sw128(0, ATOM_BYTES, 1024);
    GradWalk<F32_BK> w;
    tc::RingAt at;
    for (bool more = w.first(a, sh); more; more = w.next(a, sh)) {
        if (!wait_for<true>(&sh.acc_empty[at.s], at.phase ^ 1u, sh, a.error_word)) return;
        if (!wait_for<true>(&sh.full[at.s], at.phase, sh, a.error_word)) return;
        tc::tc_fence_after_sync();
        __syncwarp();
        const uint32_t d = sh.tmem_base + at.s * 128;
        const uint64_t da = desc + ((planes + 3 * at.s * ATOM_BYTES) >> 4), db = da + (2 * ATOM_BYTES >> 4);
        tc::mma_pair_by_warp(d, da + 2 * plane, db, idesc, 0u);
        tc::mma_pair_by_warp(d, da, db + 2 * plane, idesc, 1u);
        tc::mma_pair_by_warp(d, da + plane, db + plane, idesc, 1u);
        tc::mma_pair_by_warp(d, da + plane, db, idesc, 1u);
        tc::mma_pair_by_warp(d, da, db + plane, idesc, 1u);
        if (w.k_end - w.k0 > 16) {  // 16 rows further
            const uint64_t x = da + 128, y = db + 128;
            tc::mma_pair_by_warp(d, x + 2 * plane, y, idesc, 1u);
            tc::mma_pair_by_warp(d, x, y + 2 * plane, idesc, 1u);
            tc::mma_pair_by_warp(d, x + plane, y + plane, idesc, 1u);
            tc::mma_pair_by_warp(d, x + plane, y, idesc, 1u);
            tc::mma_pair_by_warp(d, x, y + plane, idesc, 1u);
            tc::mma_pair_by_warp(d, x, y, idesc, 1u);
        }
        tc::mma_pair_by_warp(d, da, db, idesc, 1u);
        tc::commit_pair_by_warp(&sh.empty[at.s]);
        tc::commit_pair_by_warp(&sh.acc_full[at.s]);
        at.advance(F32_STAGES);
    }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(F32_THREADS, 1) layer_wgrad_f32_kernel(const __grid_constant__ GradArgs a) {
    static_assert(F32_DYNAMIC_BYTES + sizeof(GradF32Shared) <= SMEM_MOST, "shared memory of a block");
    extern __shared__ uint8_t bytes[];
    __shared__ GradF32Shared sh;
    uint8_t* const raw = bytes + ((1024u - (tc::smem_u32(bytes) & 1023u)) & 1023u);
    const uint32_t planes = tc::smem_u32(raw) + RAW_STAGES * RAW_BYTES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int DRAINS = F32_DRAIN_WARPS;
    if (threadIdx.x == 0) {
        for (int s = 0; s < F32_STAGES; ++s) {
            tc::mbar_init(&sh.full[s], 2 * SPLIT_WARPS);
            tc::mbar_init(&sh.empty[s], 1);
            tc::mbar_init(&sh.acc_full[s], 1);
            tc::mbar_init(&sh.acc_empty[s], 2 * DRAINS);
        }
        for (int s = 0; s < RAW_STAGES; ++s) {
            tc::mbar_init(&sh.raw_full[s], 1);
            tc::mbar_init(&sh.raw_free[s], SPLIT_WARPS);
        }
        sh.abort = 0;
        tc::fence_barrier_init();
    }
    if (warp == DRAINS) {
        tc::tmem_alloc_pair(&sh.tmem_base, 512);
        tc::tmem_relinquish_pair();
    }
    wait_for_kernel_before();
    lay_out<WEIGHT_GRADIENT, F32_THREADS, F32_BK>(a, sh);
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();  // both blocks' barriers and tensor memory exist before either is signalled
    tc::tc_fence_after_sync();
    const int rank = (int)tc::cluster_rank();
    if (warp < DRAINS) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SUMS_REGISTERS));
        grad_drain<F32_BK, F32_BK, F32_STAGES, 128, F32_DRAIN_WARPS / 4, true>(a, sh, rank, [](const GradWalk<F32_BK>&, int) { return true; }, [](const GradWalk<F32_BK>&) {});
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F32_OTHER_REGISTERS));
        if (warp == DRAINS && rank == 0) grad_f32_multiplier(a, sh, planes);
        if (warp == DRAINS + 1 && lane == 0) grad_f32_producer(a, sh, raw, rank);
        if (warp >= DRAINS + 4) grad_f32_splitter(a, sh, tc::smem_u32(raw), planes, rank, warp - DRAINS - 4, lane);
    }
    __syncwarp();
    if (*reinterpret_cast<volatile int*>(&sh.abort)) __nanosleep(1000000);  // a wait ran out: copies and MMAs under way land before the block ends
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();  // neither block leaves while the other may still signal it or read its operands
    if (warp == DRAINS) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc_pair(sh.tmem_base, 512);
    }
}

// The slots of every part added up in order, four neighbouring values a thread; blocks take many, because each has to number the tiles first (a block
// for every 128 values took 105 us for 16 parts of 256 x 1,024).
template <class O>
__global__ void __launch_bounds__(256) layer_wgrad_reduce_kernel(const __grid_constant__ GradArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    __shared__ float4 red[8][32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.n ? *a.chunk_rows : 1, a.tiles, tile_start, warp_sums, a.span);
    auto add = [](float4& s, const float4 v) {
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
    };
    const int part = blockIdx.y, from = a.all_parts ? 0 : tile_start[part], count = tile_start[a.all_parts ? a.G : part + 1] - from, quads = (int)a.ldo / 4;
    const int64_t slot = (a.d_in + a.sum_rows) * a.ldo;
    const int all = a.rows * quads;
    const float* const slots = a.slots + from * slot + a.first_row * a.ldo;
    auto put = [&](int i, float4 s) {
        const int at = i / quads, row = a.first_row + at, col = 4 * (i - at * quads);
        O* to = row < a.d_in ? static_cast<O*>(a.to_w) + part * a.dw_stride + (int64_t)row * a.real_out : static_cast<O*>(a.to_b) + part * a.db_stride;
        const int second = a.d_out > a.width && col >= a.width ? 1 : 0, c = col - second * a.width;  // (of two halves each is a multiple of 8)
        to += second * a.real_width + c;
        if (c < a.real_width) to[0] = from_f32<O>(s.x);
        if (c + 1 < a.real_width) to[1] = from_f32<O>(s.y);
        if (c + 2 < a.real_width) to[2] = from_f32<O>(s.z);
        if (c + 3 < a.real_width) to[3] = from_f32<O>(s.w);
    };
    // a quad's sums over every `step`-th slot from `first` on; the bias's over the shares of the rows, too
    auto sum = [&](int i, int first, int step) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        const int shares = i >= (a.d_in - a.first_row) * quads ? a.sum_rows : 1;
        for (int k = 0; k < shares; ++k) {
            const float* p = slots + first * slot + 4 * (int64_t)i + k * a.ldo;
#pragma unroll 4
            for (int t = first; t < count; t += step, p += step * slot) add(s, *reinterpret_cast<const float4*>(p));
        }
        return s;
    };
    // where there are many slots and few quads, eight warps share the slots of 32 quads; otherwise every thread has a quad of its own
    if (count >= 8 && (int)gridDim.x * 32 >= all) {
        const int lane = threadIdx.x & 31, share = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < all) s = sum(i, share, 8);
        red[share][lane] = s;
        __syncthreads();
        if (share || i >= all) return;
#pragma unroll
        for (int k = 1; k < 8; ++k) add(s, red[k][lane]);
        put(i, s);
    } else {
        for (int i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) put(i, sum(i, 0, 1));
    }
}

}  // namespace

int32_t layer_dw(rtma_ctx* ctx, const char* who, const rtma_layer_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx, const void* dZ,
                 int64_t lddz, int width, void* dW, int64_t dw_stride, void* db, int64_t db_stride, bool sums, size_t at, size_t* scratch, cudaStream_t stream) {
    const int halves = d->gated ? 2 : 1, d_in = d->d_in, d_out = halves * width, real_out = halves * d->d_out;
    const int64_t weights = (int64_t)d_in * real_out;
    const bool bf16 = d->dtype == RTMA_BF16, f32 = d->dtype == RTMA_F32;
    auto overlap = [G](int64_t stride, int64_t size) { return G > 1 && stride && stride < size && stride > -size; };
    if (overlap(dw_stride, weights) || (db && overlap(db_stride, real_out))) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: gradients of the parts overlap", who);
    // One gradient for all parts: their rows are cut into chunks as one.  Of weights and bias only one: cut part by part, and only what is for all of them
    // is added up over all.
    const bool mixed = G > 1 && db && sums && (dw_stride == 0) != (db_stride == 0), shared = G > 1 && dw_stride == 0 && !mixed;
    GradArgs a{};
    a.error_word = ctx->error_word;
    a.offsets = offsets; a.n = n;
    a.G = shared ? 1 : G;
    a.span = shared ? G : 1;
    a.d_in = d_in; a.d_out = d_out;
    // MMAs of either orientation, in columns of the right operand
    auto tile = [](int columns) { return columns > LEFT / 2 ? LEFT : LEFT / 2; };  // (of few columns both blocks bring a half: 300,000 x 100 x 47 45 -> 43 us)
    const int64_t as_left = ceil_div(d_in, tile(d_in)) * ceil_div(d_out, 32), swapped = ceil_div(d_out, tile(d_out)) * ceil_div(d_in, 32);
    a.swapped = swapped <= as_left;
    a.left = a.swapped ? d_out : d_in; a.right = a.swapped ? d_in : d_out;
    a.A = a.swapped ? dZ : X; a.lda = a.swapped ? lddz : ldx;
    a.B = a.swapped ? X : dZ; a.ldb = a.swapped ? ldx : lddz;
    a.left_half = tile(a.left) / 2;
    a.m_tiles = (int)ceil_div(a.left, 2 * a.left_half);
    const int widest = f32 ? 2 * F32_HALF : 256;  // columns of the right operand in a tile
    a.n_tiles = (int)ceil_div(a.right, widest);
    a.half = (int)ceil_div(ceil_div(a.right, a.n_tiles), 32) * 16;
    a.n_tiles = (int)ceil_div(a.right, 2 * a.half);
    const int pairs = ctx->sm_count / 2;
    a.tile_rows = 256;
    a.tiles = std::min(std::max<int64_t>(a.G, (int64_t)DW_WAVES * pairs / ((int64_t)a.m_tiles * a.n_tiles)), n / a.tile_rows + a.G);
    a.ldo = ceil_div(d_out, 8) * 8;
    a.width = width; a.real_width = d->d_out; a.real_out = real_out;
    a.to_w = dW; a.dw_stride = dw_stride; a.to_b = db; a.db_stride = db_stride;
    a.sums = db && sums;
    a.sum_rows = f32 ? 4 : 2;
    const size_t bytes = at + 256 + sizeof(float) * (size_t)a.tiles * (d_in + a.sum_rows) * a.ldo;
    if (scratch) {
        *scratch = bytes;
        return RTMA_OK;
    }
    RTMA_TRY(prepare_row_call(ctx, bytes, stream));
    a.chunk_rows = reinterpret_cast<int32_t*>(ctx->arena + at);
    a.slots = reinterpret_cast<float*>(ctx->arena + at + 256);
    if (n > 0) {
        const int64_t tiles = a.tiles * a.m_tiles * a.n_tiles;
        if (tiles >= (int64_t(1) << 30)) return rtma_fail(ctx, RTMA_ERR_OVERFLOW, "%s: %lld tiles", who, (long long)tiles);
        // fp32 rows as twice as many 16-bit values, in boxes of 32 of them and as many rows
        const int values = f32 ? 2 : 1, box = f32 ? F32_BK : BK;
        if (!make_tensor_map_16bit(&a.map_a, f32 || bf16, a.A, 1, n, values * (uint64_t)a.left, values * a.lda, values * n * a.lda, box) ||
            !make_tensor_map_16bit(&a.map_b, f32 || bf16, a.B, 1, n, values * (uint64_t)a.right, values * a.ldb, values * n * a.ldb, box))
            return rtma_fail(ctx, RTMA_ERR_CUDA, "%s: no tensor map for rows of %d and %d values", who, d_in, d_out);
        void (*kernel)(GradArgs) = f32 ? layer_wgrad_f32_kernel : bf16 ? layer_wgrad_kernel<__nv_bfloat16> : layer_wgrad_kernel<__half>;
        const int bytes_of = f32 ? F32_DYNAMIC_BYTES : DYNAMIC_BYTES;
        bool& configured = ctx->layer_configured[32 + d->dtype];
        if (!configured) {
            RTMA_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes_of));
            configured = true;
        }
        KernelScope ks(ctx, KC_GEMM_WGRAD, stream);
        launch_kernel(kernel, (unsigned)(2 * std::min<int64_t>(tiles, pairs)), f32 ? F32_THREADS : THREADS, bytes_of, stream, a);
        RTMA_LAUNCH_CHECK(ctx);
    }
    KernelScope ks(ctx, KC_REDUCE_SGD, stream);
    void (*reduce)(GradArgs) = d->grad_dtype == RTMA_F32 ? layer_wgrad_reduce_kernel<float> : bf16 ? layer_wgrad_reduce_kernel<__nv_bfloat16> : layer_wgrad_reduce_kernel<__half>;
    auto add_up = [&](int first_row, int rows, bool all_parts) {
        a.first_row = first_row; a.rows = rows; a.all_parts = all_parts;
        const int parts = all_parts ? 1 : a.G;
        launch_kernel(reduce, dim3((unsigned)std::min<int64_t>(ceil_div(rows * a.ldo / 4, 32), std::max(1, 8 * ctx->sm_count / parts)), (unsigned)parts), 256, 0, stream, a);
    };
    if (!mixed) {
        add_up(0, d_in + (a.sums ? 1 : 0), false);
    } else {
        add_up(0, d_in, dw_stride == 0);
        RTMA_LAUNCH_CHECK(ctx);
        add_up(d_in, 1, db_stride == 0);
    }
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}
