// Whole layers (layer.cu) on fp32 rows, and the gradient of their rows.
//
// A value is split into three bf16 numbers and a product is six MMAs; 32 terms start a fresh accumulator, the five small products first, and are
// then added up in registers, rounded to nearest (grouped_split.cu says why).  Pairs of blocks (MMAs of 256 rows by up to 256 columns), each step
// with warps of its own, so that the MMAs wait for none of them:
//   one warp   bulk-tensor loads of the rows as they are (three stages) and of the matrix's planes, which are split once a call (two)
//   six warps  split a stage's rows into planes (two took twice the MMAs' time)
//   one warp   MMAs
//   16 warps   take 64 columns of 32 rows of the accumulator after every stage, and a finished tile through the layer, 16 columns at a time
// 200,000 x 256 -> 256 with a residual branch 170 us, of which the MMAs take 105 (1.5 PFLOP/s of bf16): a tile's results and what is read beside them
// leave and come in one go, while the MMAs can be two stages ahead only.  All steps in turn by the same warps, two blocks on an SM as in
// grouped_split.cu, took 327.  Spilled, by the warps that drain: 120 to 304 bytes a thread, once a tile.
//
// The two matrices of a gated layer lie by turns of 32 columns in the planes: the 64 columns of a warp are then 32 results, and a lane has both
// factors of each of its own.
#include <algorithm>

#include "layer.cuh"
#include "split.cuh"

RTMA_BOUNDS_TU()

namespace {

using namespace grouped;

constexpr int BM = PAIR_BM, BK = 32, DRAIN_WARPS = 16, SPLIT_WARPS = 6, THREADS = 32 * (DRAIN_WARPS + 2 + SPLIT_WARPS);
constexpr int RAW_STAGES = 3, RAW_BYTES = BM * BK * 4, STAGES = 2;
constexpr int A_PLANE = BM * BK * 2, W_ATOM = 3 * 64 * BK * 2;  // a plane of the rows; three planes of 64 columns
constexpr int A_BYTES = 3 * A_PLANE, W_BYTES = 2 * W_ATOM, SLAB = 32 * 64, SLABS = 2;
constexpr int DYNAMIC_BYTES = 1024 + RAW_STAGES * RAW_BYTES + STAGES * (A_BYTES + W_BYTES) + DRAIN_WARPS * SLABS * SLAB;
constexpr int DRAIN_REGISTERS = 96, OTHER_REGISTERS = 48;  // 512 x 96 + 256 x 48 = 768 x 80

struct F32Shared : Shared {
    uint64_t raw_full[RAW_STAGES], raw_free[RAW_STAGES];
    uint64_t side[DRAIN_WARPS][SLABS];  // slabs that rows read beside the sums have come to
};

// The stages of a pair's tiles.
struct StageWalk {
    PairWalk w;
    int k, blocks;
    __device__ __forceinline__ bool open(const LayerArgs& a, const Shared& sh) {
        blocks = (a.d_in + BK - 1) / BK;
        k = 0;
        return w.open(a, sh);
    }
    __device__ __forceinline__ bool next(const Shared& sh) {
        if (++k < blocks) return true;
        k = 0;
        return w.next(sh);
    }
};

__device__ __forceinline__ void f32_producer(const LayerArgs& a, F32Shared& sh, uint8_t* raw, uint8_t* planes, int rank) {
    tc::prefetch_tensormap(&a.map_a);
    tc::prefetch_tensormap(&a.map_b);
    const int atoms = (a.half + 63) / 64, col = ((blockIdx.x >> 1) % a.n_tiles) * 2 * a.half + rank * a.half;
    StageWalk w, ahead;
    bool more = w.open(a, sh), ahead_more = more, ok = true;
    ahead = w;
    tc::RingAt at, raw_at;
    auto bring_rows = [&]() {  // two stages ahead of the planes
        if (!ahead_more) return true;
        if (!wait_for(&sh.raw_free[raw_at.s], raw_at.phase ^ 1u, sh, a.error_word)) return false;
        tc::mbar_arrive_expect_tx(&sh.raw_full[raw_at.s], RAW_BYTES);
        tc::tma_load_3d(raw + raw_at.s * RAW_BYTES, &a.map_a, &sh.raw_full[raw_at.s], 2 * BK * ahead.k, (int)ahead.w.first_row + BM * rank, 0);
        raw_at.advance(RAW_STAGES);
        ahead_more = ahead.next(sh);
        return true;
    };
    ok = bring_rows() && bring_rows();
    int filled = 0;
    for (; more && ok; more = w.next(sh)) {
        if (!wait_for<true>(&sh.empty[at.s], at.phase ^ 1u, sh, a.error_word)) {
            ok = false;
            break;
        }
        filled = min(filled + 1, STAGES);
        const uint32_t bar = tc::leader_addr(&sh.full[at.s]);
        if (rank == 0) tc::mbar_arrive_expect_tx(&sh.full[at.s], 2 * atoms * W_ATOM);
        for (int i = 0; i < atoms; ++i) tc::tma_load_3d_pair(planes + at.s * W_BYTES + i * W_ATOM, &a.map_b, bar, col + 64 * i, BK * w.k, a.w_stride ? 3 * w.w.part : 0);
        at.advance(STAGES);
        ok = bring_rows();
    }
    // No signal stays under way: every stage filled is waited for until both blocks have it back or, after a give-up, until its loads have
    // landed (the first block, for both).
    for (int i = 0; i < filled; ++i) {
        const int back = filled - i, s = (at.s - back + STAGES) % STAGES;
        const uint32_t parity = s < at.s ? at.phase : at.phase ^ 1u;
        if (!ok || !wait_for<true>(&sh.empty[s], parity, sh, a.error_word)) {
            ok = false;
            if (rank == 0)
                for (uint32_t k = 0; k < (1u << 14) && !tc::mbar_try_wait_cluster(&sh.full[s], parity); ++k) {}
        }
    }
}

// A warp's share of a stage's rows: units of eight terms.
__device__ __forceinline__ void f32_splitter(const LayerArgs& a, F32Shared& sh, uint32_t raw, uint32_t planes, int which, int lane) {
    StageWalk w;
    tc::RingAt at, raw_at;
    for (bool more = w.open(a, sh); more; more = w.next(sh)) {
        if (!wait_for(&sh.raw_full[raw_at.s], raw_at.phase, sh, a.error_word)) return;
        if (!wait_for<true>(&sh.empty[at.s], at.phase ^ 1u, sh, a.error_word)) return;
        __syncwarp();
        const uint32_t from = raw + raw_at.s * RAW_BYTES, to = planes + at.s * A_BYTES;
#pragma unroll
        for (int i = 0; i < (BM * 4 + 32 * SPLIT_WARPS - 1) / (32 * SPLIT_WARPS); ++i) {
            const int j = 32 * (SPLIT_WARPS * i + which) + lane, row = j >> 2, unit = j & 3;
            if (32 * SPLIT_WARPS * (i + 1) > BM * 4 && j >= BM * 4) break;  // (a warp as a whole)
            const uint4 lo = load_16(from + row * 128 + (((2 * unit) ^ (row & 7)) << 4)), hi = load_16(from + row * 128 + (((2 * unit + 1) ^ (row & 7)) << 4));
            const uint32_t v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            uint4 p[3];
            split_eight(v, p);
#pragma unroll
            for (int k = 0; k < 3; ++k) store_16(to + k * A_PLANE + row * 64 + ((unit ^ (row >> 1 & 3)) << 4), p[k]);
        }
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            tc::mbar_arrive(&sh.raw_free[raw_at.s]);
            tc::mbar_arrive_written(tc::leader_addr(&sh.full[at.s]));
        }
        raw_at.advance(RAW_STAGES);
        at.advance(STAGES);
    }
}

__device__ __forceinline__ uint64_t describe(uint32_t lbo, uint32_t sbo, bool narrow) {  // narrow: 64-byte swizzle
    return ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(sbo >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)(narrow ? 4 : 2) << 61);
}

__device__ __forceinline__ void f32_multiplier(const LayerArgs& a, F32Shared& sh, uint32_t rows, uint32_t planes) {
    const uint32_t idesc = tc::idesc_bf16(2 * BM, 2 * a.half, false, true);
    constexpr uint32_t ap = A_PLANE >> 4, wp = 64 * BK * 2 >> 4;  // from one plane to the next
    const Turns turns(a.half);
    StageWalk w;
    tc::RingAt at, acc;
    for (bool more = w.open(a, sh); more; more = w.next(sh)) {
        if (!wait_for<true>(&sh.acc_empty[acc.s], acc.phase ^ 1u, sh, a.error_word)) return;
        if (!wait_for<true>(&sh.full[at.s], at.phase, sh, a.error_word)) return;
        tc::tc_fence_after_sync();
        __syncwarp();
        const uint32_t d = sh.tmem_base + acc.s * turns.spacing;
        const uint64_t da = describe(16, 512, true) + ((rows + at.s * A_BYTES) >> 4), db = describe(W_ATOM, 1024, false) + ((planes + at.s * W_BYTES) >> 4);
        const bool two = a.d_in - BK * w.k > 16;
        tc::mma_pair_by_warp(d, da + 2 * ap, db, idesc, 0u);
        tc::mma_pair_by_warp(d, da, db + 2 * wp, idesc, 1u);
        tc::mma_pair_by_warp(d, da + ap, db + wp, idesc, 1u);
        tc::mma_pair_by_warp(d, da + ap, db, idesc, 1u);
        tc::mma_pair_by_warp(d, da, db + wp, idesc, 1u);
        if (two) {  // 16 terms further: 32 bytes of a row, 16 rows of the matrix
            const uint64_t x = da + 2, y = db + 128;
            tc::mma_pair_by_warp(d, x + 2 * ap, y, idesc, 1u);
            tc::mma_pair_by_warp(d, x, y + 2 * wp, idesc, 1u);
            tc::mma_pair_by_warp(d, x + ap, y + wp, idesc, 1u);
            tc::mma_pair_by_warp(d, x + ap, y, idesc, 1u);
            tc::mma_pair_by_warp(d, x, y + wp, idesc, 1u);
            tc::mma_pair_by_warp(d, x, y, idesc, 1u);
        }
        tc::mma_pair_by_warp(d, da, db, idesc, 1u);
        tc::commit_pair_by_warp(&sh.empty[at.s]);
        tc::commit_pair_by_warp(&sh.acc_full[acc.s]);
        acc.advance(turns.buffers);
        at.advance(STAGES);
    }
}

template <bool GATED, bool GRADIENT, int ACT, bool BESIDE>
__device__ __forceinline__ void f32_drain(const LayerArgs& a, F32Shared& sh, uint32_t slabs, int rank) {
    typedef Outlet<float, SLABS> Out;
    constexpr int ITEMS = GATED ? 2 : 4;  // of 16 results a row
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3;
    const Turns turns(a.half);
    const int slice = (warp >> 2) % turns.slices, group = (warp >> 2) / turns.slices;
    slabs += warp * SLABS * SLAB;
    LayerBias bias{sh.bias + 64 * warp};
    uint64_t* const side = sh.side[warp];
    const uint32_t tmem = sh.tmem_base + ((uint32_t)(32 * quarter) << 16) + 64 * slice;
    const int pair = blockIdx.x >> 1, place = pair / a.n_tiles, n0 = (pair - place * a.n_tiles) * 2 * a.half + 64 * slice;  // first column of the planes
    const int here = min(64, 2 * a.half - 64 * slice), c0 = GATED ? n0 / 2 : n0, above = BM * rank + 32 * quarter;
    const int results = here <= 0 ? 0 : max(0, min(GATED ? here / 2 : here, a.width - c0)), mine = (results + 15) / 16;
    PairWalk w;
    tc::RingAt acc;
    uint32_t n = 0;  // slabs of 16 results that this warp has been through
    float slope = 0.f, slope_sum = 0.f;
    int part = -1, turn = 0;
    for (bool more = w.open(a, sh); more; more = w.next(sh), turn = turn + 1 & turns.groups - 1) {
        const int rows = min(32, w.left - above);
        const int64_t row0 = w.first_row + above;
        const bool some = rows > 0 && mine > 0 && turn == group;
        // the rows beside 16 results, into slab (n + j) & 1, whose last store has to have been read
        auto request = [&](int j) {
            if (j >= mine || lane) return;
            uint64_t* bar = &side[(n + j) & 1];
            tc::mbar_arrive_expect_tx(bar, SLAB);
            asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                         ::"r"(slabs + ((n + j) & 1) * SLAB), "l"(reinterpret_cast<uint64_t>(&a.map_side)), "r"(tc::smem_u32(bar)), "r"(c0 + 16 * j), "r"((int)row0)
                         : "memory");
        };
        if (BESIDE && some) {
            if (lane == 0) tc::tma_store_wait_read_but<0>();
            __syncwarp();
            request(0);
            request(1);
            if (lane >= 2 && lane < mine)  // the others come to the L2 cache meanwhile
                asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(&a.map_side)), "r"(c0 + 16 * lane), "r"((int)row0) : "memory");
        }
        if (w.part != part) {
            part = w.part;
            bias.fetch(a, part, n0, mine ? 2 : 0, lane, static_cast<const float*>(nullptr), [&](int i) { return GATED ? c0 + (i ? a.bias_up : 0) : c0 + 32 * i; },
                       [&](int i) { return a.bias_width - c0 - (GATED ? 0 : 32 * i); });
            if (ACT == RTMA_ACT_PRELU) slope = __ldg(a.slope + part * a.slope_stride);
        }
        f2 total[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) total[j] = pack2(0.f, 0.f);
        for (int k = 0; k < a.d_in; k += BK) {
            if (!wait_for<true>(&sh.acc_full[acc.s], acc.phase, sh, a.error_word)) return;
            __syncwarp();
            tc::tc_fence_after_sync();
            if (some) {
                const uint32_t from = tmem + acc.s * turns.spacing;
                uint32_t x[2][8];
                tc::tmem_load_issue_8(from, x[0]);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    tc::tmem_load_wait_8(x[q & 1]);
                    if (q < 7) tc::tmem_load_issue_8(from + 8 * (q + 1), x[(q + 1) & 1]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) total[4 * q + j] = add2(total[4 * q + j], pack2(__uint_as_float(x[q & 1][2 * j]), __uint_as_float(x[q & 1][2 * j + 1])));
                }
            }
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive_remote(tc::leader_addr(&sh.acc_empty[acc.s]));  // (a pair's warps all report to the first block)
            acc.advance(turns.buffers);
        }
        if (some) {
            float ds = 0.f;
            auto store = [&](int j, uint32_t slab, int second) {
                const int c = c0 + 16 * j, cols = min(16, results - 16 * j), at = second * a.width + c;
                const bool whole = c + cols == a.width && a.width % 4 == 0 && (second || !(GATED && GRADIENT)), aligned = !second || a.width % 4 == 0;
                Out outlet{0};
                if (BESIDE && !(a.vo && aligned && rows == 32 && (cols == 16 || whole))) tc::fence_proxy_async_smem();  // (not a bulk store: the slab is written by one next)
                outlet.close(a, slab, row0, at, rows, cols, whole, static_cast<float*>(a.out) + row0 * a.ldo + at, a.ldo, lane, aligned);
            };
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) {
                if (j >= mine) break;
                const uint32_t slab = slabs + ((n + j) & 1) * SLAB;
                if constexpr (BESIDE) {
                    if (!wait_for(&side[(n + j) & 1], (n + j) >> 1 & 1u, sh, a.error_word)) return;
                } else {
                    if (lane == 0) tc::tma_store_wait_read_but<1>();
                }
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    f2 z[4], y[4], d[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        z[i] = total[8 * j + 4 * q + i];
                        if constexpr (GATED) y[i] = total[16 + 8 * j + 4 * q + i];
                    }
                    if constexpr (BESIDE) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint4 x = load_16(slab + lane * 64 + (((2 * q + h) ^ Out::swizzle(lane)) << 4));
                            d[2 * h] = pack2(__uint_as_float(x.x), __uint_as_float(x.y));
                            d[2 * h + 1] = pack2(__uint_as_float(x.z), __uint_as_float(x.w));
                        }
                    }
                    ds += eight_results<GATED, GRADIENT>(ACT, BESIDE, bias, 16 * j + 8 * q, 32 + 16 * j + 8 * q, slope, a.slope_slots != nullptr, results - 16 * j - 8 * q, z, y, d);
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        unpack2(z[i], v[2 * i], v[2 * i + 1]);
                        if constexpr (GATED && GRADIENT) total[16 + 8 * j + 4 * q + i] = y[i];
                    }
                    Out::piece(slab, lane, 2 * q, Out::pack_piece(v));
                    Out::piece(slab, lane, 2 * q + 1, Out::pack_piece(v + 4));
                    if (BESIDE && !GATED && q == 0 && j >= 1 && j < ITEMS - 1) {  // the rows beside the next 16 results, into the slab that the last ones have left
                        if (lane == 0) tc::tma_store_wait_read_but<0>();
                        __syncwarp();
                        request(j + 1);
                    }
                }
                store(j, slab, 0);
            }
            if constexpr (GATED && GRADIENT) {  // the second halves, kept until the slabs are free again
                if (lane == 0) tc::tma_store_wait_read_but<0>();
                __syncwarp();
#pragma unroll
                for (int j = 0; j < ITEMS; ++j) {
                    if (j >= mine) break;
                    const uint32_t slab = slabs + ((n + j) & 1) * SLAB;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[4];
                        unpack2(total[16 + 8 * j + 2 * q], v[0], v[1]);
                        unpack2(total[16 + 8 * j + 2 * q + 1], v[2], v[3]);
                        Out::piece(slab, lane, q, Out::pack_piece(v));
                    }
                    store(j, slab, 1);
                }
            }
            n += mine;
            if (ACT == RTMA_ACT_PRELU && lane < rows) slope_sum += ds;  // (what the accumulator has for rows that are not there may be anything)
        }
        if (GRADIENT && ACT == RTMA_ACT_PRELU && a.slope_slots && w.part_ends(sh)) {
            for (int o = 16; o > 0; o >>= 1) slope_sum += __shfl_xor_sync(0xffffffffu, slope_sum, o);
            const int64_t slot = 8 * (int64_t)(place + part) + 4 * rank + quarter;
            if (lane == 0) a.slope_slots[(slot * a.n_tiles + (pair - place * a.n_tiles)) * 4 + (warp >> 2)] = slope_sum;
            slope_sum = 0.f;
        }
    }
    if (lane == 0) tc::tma_store_wait_all();
}

template <bool GATED, bool GRADIENT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) layer_f32_kernel(const __grid_constant__ LayerArgs a) {
    static_assert(DYNAMIC_BYTES + sizeof(F32Shared) <= SMEM_MOST, "shared memory of a block");
    extern __shared__ uint8_t raw_bytes[];
    __shared__ F32Shared sh;
    uint8_t* const raw = raw_bytes + ((1024u - (tc::smem_u32(raw_bytes) & 1023u)) & 1023u);
    uint8_t* const w_planes = raw + RAW_STAGES * RAW_BYTES;
    const uint32_t a_planes = tc::smem_u32(w_planes) + STAGES * W_BYTES, slabs = a_planes + STAGES * A_BYTES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x >= 32 && threadIdx.x < 32 + DRAIN_WARPS * SLABS) {
        tc::mbar_init(&sh.side[(threadIdx.x - 32) / SLABS][threadIdx.x % SLABS], 1);
        tc::fence_barrier_init();
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            tc::mbar_init(&sh.full[s], 1 + 2 * SPLIT_WARPS);  // the planes of the matrix; both blocks' rows
            tc::mbar_init(&sh.empty[s], 1);
        }
        for (int b = 0; b < MAX_ACCUMULATORS; ++b) {
            tc::mbar_init(&sh.acc_full[b], 1);
            tc::mbar_init(&sh.acc_empty[b], 2 * DRAIN_WARPS);
        }
        for (int s = 0; s < RAW_STAGES; ++s) {
            tc::mbar_init(&sh.raw_full[s], 1);
            tc::mbar_init(&sh.raw_free[s], SPLIT_WARPS);
        }
        sh.abort = 0;
        tc::fence_barrier_init();
    }
    if (warp == DRAIN_WARPS) {
        tc::tmem_alloc_pair(&sh.tmem_base, 512);
        tc::tmem_relinquish_pair();
    }
    wait_for_kernel_before();
    lay_out<FORWARD, THREADS, BK>(a, sh);
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();  // both blocks' barriers and tensor memory exist before either is signalled
    tc::tc_fence_after_sync();
    const int rank = (int)tc::cluster_rank();
    if (warp < DRAIN_WARPS) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(DRAIN_REGISTERS));
        with_activation<GRADIENT>(a, [&](auto act, auto beside) { f32_drain<GATED, GRADIENT, decltype(act)::value, decltype(beside)::value>(a, sh, slabs, rank); });
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGISTERS));
        if (warp == DRAIN_WARPS && rank == 0) f32_multiplier(a, sh, a_planes, tc::smem_u32(w_planes));
        if (warp == DRAIN_WARPS + 1 && lane == 0) f32_producer(a, sh, raw, w_planes, rank);
        if (warp >= DRAIN_WARPS + 2) f32_splitter(a, sh, tc::smem_u32(raw), a_planes, warp - DRAIN_WARPS - 2, lane);
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

struct PlanesArgs {
    const float* W;
    int64_t w_stride;
    int parts, d_in, width, halves, up, granule, ld, ldt;
    __nv_bfloat16 *planes, *transposed;
};
__global__ void __launch_bounds__(256) layer_planes_kernel(const __grid_constant__ PlanesArgs a) {
    wait_for_kernel_before();
    const int wide = a.halves * a.width;
    if (blockIdx.y == 0) {
        const int units = a.ld / 8;
        const int64_t matrix = (int64_t)a.ld * a.d_in, total = a.planes ? (int64_t)a.parts * a.d_in * units : 0;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
            const int64_t row = i / units, part = row / a.d_in, r = row - part * a.d_in;
            const int u = (int)(i - row * units);
            const int second = a.halves == 2 ? u >> 2 & 1 : 0, c = a.halves == 2 ? 32 * (u >> 3) + 8 * (u & 3) : 8 * u, valid = max(0, min(8, a.width - c));
            Eight<float> x;
            x.load(a.W + part * a.w_stride + r * wide + second * a.width + (valid ? c : 0), valid, a.granule);
            uint4 p[3];
            split_eight(reinterpret_cast<const uint32_t(&)[8]>(x.w), p);
#pragma unroll
            for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(a.planes + (3 * part + k) * matrix + r * a.ld + 8 * u) = p[k];
        }
    } else {  // neighbouring threads have neighbouring columns of the matrix, which are rows of the planes
        const int units = a.ldt / 8, rows = a.halves * a.up;
        const int64_t matrix = (int64_t)a.ldt * rows, total = (int64_t)a.parts * units * rows;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
            const int64_t run = i / rows, part = run / units;
            const int r = (int)(i - run * rows), u = (int)(run - part * units), second = r >= a.up ? 1 : 0, c = r - second * a.up;
            const float* from = a.W + part * a.w_stride + second * a.width + c;
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = c < a.width && 8 * u + j < a.d_in ? __float_as_uint(from[(int64_t)(8 * u + j) * wide]) : 0u;
            uint4 p[3];
            split_eight(v, p);
#pragma unroll
            for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(a.transposed + (3 * part + k) * matrix + (int64_t)r * a.ldt + 8 * u) = p[k];
        }
    }
}

}  // namespace

int32_t split_matrices(rtma_ctx* ctx, const float* W, int64_t w_stride, int parts, int d_in, int width, int halves, int up, void* planes, int ld, void* transposed, int ldt,
                       cudaStream_t stream) {
    PlanesArgs a{W, w_stride, parts, d_in, width, halves, up, 0, ld, ldt, static_cast<__nv_bfloat16*>(planes), static_cast<__nv_bfloat16*>(transposed)};
    a.granule = std::min({row_granule(W, (int64_t)halves * width, 4), row_granule(nullptr, w_stride, 4), row_granule(nullptr, width, 4)});
    const int64_t most = std::max((int64_t)d_in * ld, transposed ? (int64_t)halves * up * ldt : 0) / 8 * parts;
    KernelScope ks(ctx, KC_WEIGHT_PREP, stream);
    launch_kernel(layer_planes_kernel, dim3((unsigned)std::min<int64_t>(ceil_div(most, 256), 16 * ctx->sm_count), transposed ? 2 : 1), 256, 0, stream, a);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

int32_t launch_layer_f32(rtma_ctx* ctx, LayerArgs& a, bool gated, bool gradient, int cls, unsigned grid, cudaStream_t stream) {
    // rows as twice as many 16-bit values: boxes of 32 terms
    if (!make_tensor_map_16bit(&a.map_b, true, a.B, 3 * (uint64_t)(a.w_stride ? a.G : 1), a.d_in, a.ldb, a.ldb, (uint64_t)a.ldb * a.d_in, BK, 64, 3) ||
        !make_tensor_map_16bit(&a.map_a, true, a.A, 1, a.n, 2 * (uint64_t)a.d_in, 2 * a.lda, 2 * (uint64_t)a.n * a.lda, BM) ||
        (a.side && !make_store_map(&a.map_side, RTMA_F32, a.side, a.n, a.bias_width, a.lds)))
        return rtma_fail(ctx, RTMA_ERR_CUDA, "grouped layer: no tensor map for rows of %d and %d values", a.d_in, a.width);
    void (*kernel)(LayerArgs) = gated ? (gradient ? layer_f32_kernel<true, true> : layer_f32_kernel<true, false>) : gradient ? layer_f32_kernel<false, true> : layer_f32_kernel<false, false>;
    bool& configured = ctx->layer_configured[24 + (gated ? 2 : 0) + (gradient ? 1 : 0)];
    if (!configured) {
        RTMA_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, DYNAMIC_BYTES));
        configured = true;
    }
    KernelScope ks(ctx, cls, stream);
    launch_kernel(kernel, grid, THREADS, DYNAMIC_BYTES, stream, a);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}
