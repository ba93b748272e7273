// The kernel of whole layers (layer.cu) on 16-bit rows that lie on 16-byte boundaries: pairs of blocks with the matrix resident.
//
// A pair (a cluster of two, MMAs of 256 rows) keeps the columns of one tile and walks down neighbouring row tiles.  Up to 256 terms its part
// of the matrix stays in shared memory until the part changes, and only the rows stream: brought again for every tile (RESIDENT false: deeper
// contractions) the matrix is half of what comes from the L2 cache, and that is what bounds the products: 500,000 x 256 -> 2 x 512 in bf16 with
// nothing but the MMAs took 229 us, like this 205.  With all that belongs to it 240 us (1.1 PFLOP/s, of the measured burst 64 %), the first step of its
// gradient 366 (memory: 1.8 GB, 4.9 TB/s); 500,000 x 512 -> 256 with a residual branch 176 us (5.8 TB/s), first step of the gradient of 500,000 x 256 ->
// 256 145 (5.3 TB/s).
//
// Sixteen warps drain: 32 rows and 32 columns of a tile at a time, eight columns on their way from tensor memory.  What is read beside
// the accumulators (the residual branch, the result's gradient) comes by bulk-tensor loads into the same slab of shared memory that the results
// leave from; read by the lanes, each from a row of its own, it cost twice its time from memory (gradient of 500,000 x 256 -> 256: 178 us,
// 99 without these reads).
//
// Gradient: the column sums of dZ (the bias gradient) are products with ones, by mma.sync from the slab: added up by the lanes they would cost more
// than the activation (here 5 us of 367 for 500,000 x 256 -> 2 x 512, in the weight gradient's kernel, whose tensor cores are busier, 64 and more).  They
// and the slope's gradient stay in registers until the part changes, and are left in a slot of (place of the pair + part), which no two share.
#pragma once

#include "layer.cuh"

namespace {

using namespace grouped;

constexpr int BM = PAIR_BM, BK = 64;
constexpr int SUMMED_TILES = 64;     // after which the sums of columns and slopes go to their slots, so that not every tile's meet a long sum
constexpr int RESIDENT_TERMS = 256;  // of the contraction, up to which the matrix stays in shared memory

template <class T_, bool GATED_, bool GRADIENT_, bool RESIDENT_>
struct PairForm {
    typedef T_ T;
    static constexpr bool GATED = GATED_, GRADIENT = GRADIENT_, RESIDENT = RESIDENT_;
    static constexpr int DRAIN_WARPS = 16, THREADS = 32 * (DRAIN_WARPS + 4);
    static constexpr int A_BYTES = BM * 128, B_BYTES = 128 * 128;  // 64 terms of a block's rows; of its columns, 128 at most
    static constexpr int SLABS = GATED && GRADIENT ? 3 : 2;         // of a drain warp
    static constexpr int STAGE_BYTES = A_BYTES + (RESIDENT ? 0 : B_BYTES);
    static constexpr int STAGES = RESIDENT ? (SLABS == 3 ? 3 : 5) : (SLABS == 3 ? 3 : 4);
    static constexpr int RING_BYTES = STAGES * STAGE_BYTES, HELD_BYTES = RESIDENT ? RESIDENT_TERMS / BK * B_BYTES : 0;
    static constexpr int SLAB = 32 * 64, OUT_BYTES = SLABS * SLAB;
    static constexpr int DYNAMIC_BYTES = 1024 + RING_BYTES + HELD_BYTES + DRAIN_WARPS * OUT_BYTES;
};
// Registers: 640 threads at 96; 512 x 104 + 128 x 64 = 640 x 96.
constexpr int PAIR_DRAIN_REGISTERS = 104, PAIR_OTHER_REGISTERS = 64;

struct PairShared : Shared {
    uint64_t held_full, held_empty;  // the resident matrix
    uint64_t side[16][2];            // slabs that rows read beside the accumulators have come to
};

template <class F>
__device__ __forceinline__ void pair_producer(const LayerArgs& a, PairShared& sh, uint8_t* ring, uint8_t* held, int rank) {
    tc::prefetch_tensormap(&a.map_a);
    tc::prefetch_tensormap(&a.map_b);
    const int blocks = (a.d_in + BK - 1) / BK, atoms = (a.half + 63) / 64;
    const int col = ((blockIdx.x >> 1) % a.n_tiles) * (F::GATED ? a.half : 2 * a.half) + rank * (F::GATED ? a.up : a.half);
    PairWalk w;
    tc::RingAt at;
    int filled = 0, part = -1;  // stages filled, STAGES at most
    uint32_t changes = 0;
    bool ok = true;
    for (bool more = w.open(a, sh); more && ok; more = w.next(sh)) {
        const int z = a.w_stride ? w.part : 0;
        if (F::RESIDENT && w.part != part) {
            part = w.part;
            if (!wait_for<true>(&sh.held_empty, (changes & 1u) ^ 1u, sh, a.error_word)) {
                ok = false;
                break;
            }
            ++changes;
            const uint32_t bar = tc::leader_addr(&sh.held_full);
            if (rank == 0) tc::mbar_arrive_expect_tx(&sh.held_full, 2 * blocks * atoms * 2 * SLAB_BYTES);
            for (int k = 0; k < blocks; ++k)
                for (int i = 0; i < atoms; ++i) tc::tma_load_3d_pair(held + k * F::B_BYTES + i * 2 * SLAB_BYTES, &a.map_b, bar, col + 64 * i, k * BK, z);
        }
        for (int k = 0; k < blocks; ++k) {
            if (!wait_for<true>(&sh.empty[at.s], at.phase ^ 1u, sh, a.error_word)) {
                ok = false;
                break;
            }
            filled = min(filled + 1, F::STAGES);
            uint8_t* stage = ring + at.s * F::STAGE_BYTES;
            const uint32_t bar = tc::leader_addr(&sh.full[at.s]);
            if (rank == 0) tc::mbar_arrive_expect_tx(&sh.full[at.s], 2 * (F::A_BYTES + (F::RESIDENT ? 0 : atoms * 2 * SLAB_BYTES)));
            tc::tma_load_3d_pair(stage, &a.map_a, bar, k * BK, (int)w.first_row + BM * rank, 0);
            if (!F::RESIDENT)
                for (int i = 0; i < atoms; ++i) tc::tma_load_3d_pair(stage + F::A_BYTES + i * 2 * SLAB_BYTES, &a.map_b, bar, col + 64 * i, k * BK, z);
            at.advance(F::STAGES);
        }
    }
    // No signal stays under way: every stage filled is waited for until both blocks have it back or, after a give-up, until its loads have
    // landed (the first block, for both); so is the resident matrix.
    for (int n = 0; n < filled; ++n) {
        const int back = filled - n, s = (at.s - back + F::STAGES) % F::STAGES;
        const uint32_t parity = s < at.s ? at.phase : at.phase ^ 1u;
        if (!ok || !wait_for<true>(&sh.empty[s], parity, sh, a.error_word)) {
            ok = false;
            if (rank == 0)
                for (uint32_t i = 0; i < (1u << 14) && !tc::mbar_try_wait_cluster(&sh.full[s], parity); ++i) {}
        }
    }
    if (F::RESIDENT && changes && (!ok || !wait_for<true>(&sh.held_empty, (changes & 1u) ^ 1u, sh, a.error_word)) && rank == 0)
        for (uint32_t i = 0; i < (1u << 14) && !tc::mbar_try_wait_cluster(&sh.held_full, (changes & 1u) ^ 1u); ++i) {}
}

template <class F>
__device__ __forceinline__ void pair_multiplier(const LayerArgs& a, PairShared& sh, uint32_t ring, uint32_t held) {
    const int blocks = (a.d_in + BK - 1) / BK;
    const uint32_t format = std::is_same<typename F::T, __half>::value ? 0u : 1u;  // fp16 or bf16 operands, fp32 sums
    const uint32_t idesc = (1u << 4) | (format << 7) | (format << 10) | (1u << 16) | ((uint32_t)(2 * a.half >> 3) << 17) | ((uint32_t)(2 * BM >> 4) << 24);
    const uint64_t desc = tc::smem_desc_sw128(0, 2 * SLAB_BYTES, 1024);  // atoms of 64 columns lie two slabs apart
    const Turns turns = Turns::of_pairs(F::GATED, F::GRADIENT, a.half);
    PairWalk w;
    tc::RingAt at, acc;
    int part = -1;
    uint32_t changes = 0;
    for (bool more = w.open(a, sh); more; more = w.next(sh)) {
        if (F::RESIDENT && w.part != part) {
            part = w.part;
            if (!wait_for<true>(&sh.held_full, changes++ & 1u, sh, a.error_word)) return;
        }
        if (!wait_for<true>(&sh.acc_empty[acc.s], acc.phase ^ 1u, sh, a.error_word)) return;
        const uint32_t d = sh.tmem_base + acc.s * turns.spacing;
        for (int k = 0; k < blocks; ++k) {
            if (!wait_for<true>(&sh.full[at.s], at.phase, sh, a.error_word)) return;
            tc::tc_fence_after_sync();
            __syncwarp();
            const uint32_t stage = ring + at.s * F::STAGE_BYTES;
            const uint64_t da = desc + (stage >> 4), db = desc + ((F::RESIDENT ? held + k * F::B_BYTES : stage + F::A_BYTES) >> 4);
            const int steps = (min(BK, a.d_in - k * BK) + 15) >> 4;
#pragma unroll
            for (int i = 0; i < BK / 16; ++i)
                if (i < steps) tc::mma_pair_by_warp(d, da + 2 * i, db + 128 * i, idesc, i || k ? 1u : 0u);
            tc::commit_pair_by_warp(&sh.empty[at.s]);
            at.advance(F::STAGES);
        }
        tc::commit_pair_by_warp(&sh.acc_full[acc.s]);
        acc.advance(turns.buffers);
        if (F::RESIDENT && w.part_ends(sh)) tc::commit_pair_by_warp(&sh.held_empty);
    }
}

// Sums of the 32 columns of a slab over its 32 rows, added to sums: sums[m][0] of lane l is column 16 m + l / 4, sums[m][1] the one 8 behind it.  Products
// with ones; the tensor cores' accumulators, which truncate, hold no more than these 32 rows (their other halves are the same again).
template <class T>
__device__ __forceinline__ void add_columns(uint32_t slab, int lane, float (&sums)[2][2]) {
    const uint32_t one = std::is_same<T, __half>::value ? 0x3C003C00u : 0x3F803F80u;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            // four 8 x 8 blocks: columns 16 m .. + 7 and + 8 .. + 15 of rows 16 k .. + 7, then of rows + 8 .. + 15
            const int row = 16 * k + 8 * (lane >> 4) + (lane & 7), q = 2 * m + (lane >> 3 & 1);
            uint32_t x[4];
            asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                         : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                         : "r"(slab + row * 64 + ((q ^ (row >> 1 & 3)) << 4))
                         : "memory");
            if constexpr (std::is_same<T, __half>::value)
                asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %8}, {%0, %1, %2, %3};"
                             : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                             : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(one));
            else
                asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %8}, {%0, %1, %2, %3};"
                             : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                             : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(one));
        }
        sums[m][0] += c[0];
        sums[m][1] += c[2];
    }
}

// NARROW: by turns.
template <class F, int ACT, bool BESIDE, bool NARROW>
__device__ __forceinline__ void pair_drain(const LayerArgs& a, PairShared& sh, uint32_t slabs, int rank) {
    typedef typename F::T T;
    typedef Outlet<T, F::SLABS> Out;
    constexpr bool GATED = F::GATED, GRADIENT = F::GRADIENT;
    constexpr int ITEMS = GATED ? 1 : 2, PIECE = 16 / (int)sizeof(T);  // chunks of 32 columns a tile for a warp, at most
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3;
    const Turns turns = NARROW ? Turns::of_pairs(GATED, GRADIENT, a.half) : Turns(256);
    const int slice = NARROW ? (warp >> 2) % turns.slices : warp >> 2, group = NARROW ? (warp >> 2) / turns.slices : 0;
    slabs += warp * F::OUT_BYTES;
    LayerBias bias{sh.bias + 64 * warp};
    uint64_t* const side = sh.side[warp];
    const uint32_t tmem = sh.tmem_base + ((uint32_t)(32 * quarter) << 16);
    const int n0 = ((blockIdx.x >> 1) % a.n_tiles) * (GATED ? a.half : 2 * a.half);
    const int wide = GATED ? a.half : 2 * a.half, above = BM * rank + 32 * quarter;
    auto column = [&](int i) { return n0 + 32 * (slice + 4 * i); };
    auto columns = [&](int i) { return min(min(32, wide - 32 * (slice + 4 * i)), a.width - column(i)); };
    const int mine = columns(0) <= 0 ? 0 : ITEMS == 2 && columns(1) > 0 ? 2 : 1;
    PairWalk w, ahead;
    bool more = w.open(a, sh), ahead_more = more && BESIDE && mine > 0;
    ahead = w;
    const int start = w.t;
    auto is_mine = [&](const PairWalk& x) { return !NARROW || (x.t - start & turns.groups - 1) == group; };
    int ahead_item = 0;
    // The rows beside the next 32 columns that are this warp's, into slab n & 1, whose last store has to have been read.
    auto request = [&](uint32_t n) {
        while (ahead_more && (ahead.left <= above || !is_mine(ahead))) ahead_more = ahead.next(sh);  // (a tile that ends above this warp's rows)
        if (!ahead_more) return;
        if (lane == 0) {
            uint64_t* bar = &side[n & 1];
            tc::mbar_arrive_expect_tx(bar, F::SLAB);
            asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                         ::"r"(slabs + (n & 1) * F::SLAB), "l"(reinterpret_cast<uint64_t>(&a.map_side)), "r"(tc::smem_u32(bar)), "r"(column(ahead_item)), "r"((int)ahead.first_row + above)
                         : "memory");
        }
        if (++ahead_item >= mine) {
            ahead_item = 0;
            ahead_more = ahead.next(sh);
        }
    };
    uint32_t n = 0;  // 32 columns that this warp has been through
    request(0);
    tc::RingAt acc;
    float slope = 0.f, slope_sum = 0.f, sums[GRADIENT ? 2 : 1][2][2];
    int part = -1;
    auto clear = [&]() {
        slope_sum = 0.f;
        if constexpr (GRADIENT)
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[i >> 2][i >> 1 & 1][i & 1] = 0.f;
    };
    clear();
    for (; more; more = w.next(sh)) {
        const int rows = min(32, w.left - above);
        const int64_t row0 = w.first_row + above;
        if (w.part != part) {
            part = w.part;
            bias.fetch(a, part, n0, GATED ? 2 * mine : mine, lane, static_cast<const T*>(nullptr), [&](int i) { return GATED ? column(0) + (i ? a.bias_up : 0) : column(i); },
                       [&](int i) { return min(GATED ? columns(0) : columns(i), a.bias_width - (GATED ? column(0) : column(i))); });
            if (ACT == RTMA_ACT_PRELU) slope = __ldg(a.slope + part * a.slope_stride);
        }
        if (!wait_for<true>(&sh.acc_full[acc.s], acc.phase, sh, a.error_word)) return;
        __syncwarp();
        tc::tc_fence_after_sync();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (rows <= 0 || i >= mine || !is_mine(w)) break;
            const int c = column(i), cols = columns(i);
            const uint32_t from = tmem + acc.s * turns.spacing + 32 * (slice + 4 * i);
            const uint32_t slab = slabs + (n & 1) * F::SLAB, other = slabs + 2 * F::SLAB;
            uint32_t x[2][8], x2[2][8];
            tc::tmem_load_issue_8(from, x[0]);
            if constexpr (GATED) tc::tmem_load_issue_8(from + a.half, x2[0]);
            if constexpr (BESIDE) {
                if (!wait_for(&side[n & 1], n >> 1 & 1u, sh, a.error_word)) return;
            } else {
                if (lane == 0) tc::tma_store_wait_read_but<1>();
            }
            __syncwarp();
            float ds = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                tc::tmem_load_wait_8(x[q & 1]);
                if constexpr (GATED) tc::tmem_load_wait_8(x2[q & 1]);
                if (q < 3) {
                    tc::tmem_load_issue_8(from + 8 * (q + 1), x[(q + 1) & 1]);
                    if constexpr (GATED) tc::tmem_load_issue_8(from + a.half + 8 * (q + 1), x2[(q + 1) & 1]);
                }
                f2 z[4], y[4], d[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    z[k] = pack2(__uint_as_float(x[q & 1][2 * k]), __uint_as_float(x[q & 1][2 * k + 1]));
                    if constexpr (GATED) y[k] = pack2(__uint_as_float(x2[q & 1][2 * k]), __uint_as_float(x2[q & 1][2 * k + 1]));
                }
                if constexpr (BESIDE) {
                    Eight<T> e;
                    e.w[0] = load_16(slab + lane * 64 + ((q ^ Out::swizzle(lane)) << 4));
                    pairs_of(e, d);
                }
                ds += eight_results<GATED, GRADIENT>(ACT, BESIDE, bias, 32 * i + 8 * q, 32 + 8 * q, slope, a.slope_slots != nullptr, cols - 8 * q, z, y, d);
                float v[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) unpack2(z[k], v[2 * k], v[2 * k + 1]);
                uint4 p = Out::pack_piece(v);
                if (GRADIENT && rows < 32 && lane >= rows) p = make_uint4(0u, 0u, 0u, 0u);  // (what the accumulator has there may be anything, and is summed)
                Out::piece(slab, lane, q, p);
                if constexpr (GATED && GRADIENT) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) unpack2(y[k], v[2 * k], v[2 * k + 1]);
                    if (q == 0) {  // the last second half has been read
                        if (lane == 0) tc::tma_store_wait_read_but<0>();
                        __syncwarp();
                    }
                    p = Out::pack_piece(v);
                    if (rows < 32 && lane >= rows) p = make_uint4(0u, 0u, 0u, 0u);
                    Out::piece(other, lane, q, p);
                }
                if (BESIDE && q == 0) {  // what comes next, into the slab that the columns before these have left
                    if (!(GATED && GRADIENT)) {
                        if (lane == 0) tc::tma_store_wait_read_but<0>();
                        __syncwarp();
                    }
                    request(n + 1);
                }
            }
            if (ACT == RTMA_ACT_PRELU && lane < rows) slope_sum += ds;
            T* const out = static_cast<T*>(a.out) + row0 * a.ldo + c;
            const bool whole = c + cols == a.width && a.width % PIECE == 0;
            Out outlet{0};
            if (BESIDE && !(a.vo && rows == 32 && (cols == 32 || whole))) tc::fence_proxy_async_smem();  // (not a bulk store: the slab is written by one next)
            if constexpr (GATED && GRADIENT) {
                outlet.close(a, slab, row0, c, rows, cols, false, out, a.ldo, lane);
                outlet.close(a, other, row0, a.width + c, rows, cols, whole, out + a.width, a.ldo, lane, a.width % PIECE == 0);
                if (a.column_slots) {
                    add_columns<T>(slab, lane, sums[0]);
                    add_columns<T>(other, lane, sums[1]);
                }
            } else {
                outlet.close(a, slab, row0, c, rows, cols, whole, out, a.ldo, lane);
                if constexpr (GRADIENT)
                    if (a.column_slots) add_columns<T>(slab, lane, sums[i]);
            }
            ++n;
        }
        tc::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_remote(tc::leader_addr(&sh.acc_empty[acc.s]));  // (a pair's warps all report to the first block)
        acc.advance(turns.buffers);
        if (GRADIENT && (w.part_ends(sh) || w.t % SUMMED_TILES == SUMMED_TILES - 1)) {
            const int pair = blockIdx.x >> 1, place = pair / a.n_tiles;
            // the part's first tile here; again: the slots hold sums of tiles before these
            const int first = max((int)((int64_t)sh.tile_start[a.G] * place / a.places), sh.tile_start[part]);
            const bool again = first / SUMMED_TILES < w.t / SUMMED_TILES;
            const int64_t slot = 8 * (int64_t)(place + part) + 4 * rank + quarter;  // (of the first group)
            if (a.column_slots) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if ((lane & 3) || (GATED ? mine < 1 : i >= mine)) continue;
                    float* const to = a.column_slots + (group * a.slots_up + slot) * a.columns + (GATED ? column(0) + (i ? a.width : 0) : column(i));
                    const int cols = GATED ? columns(0) : columns(i);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int j = 8 * k + (lane >> 2);
                        if (j < cols) to[j] = sums[i][k >> 1][k & 1] + (again ? to[j] : 0.f);
                    }
                }
            }
            if (ACT == RTMA_ACT_PRELU && a.slope_slots) {
                for (int o = 16; o > 0; o >>= 1) slope_sum += __shfl_xor_sync(0xffffffffu, slope_sum, o);
                float* const to = a.slope_slots + (slot * a.n_tiles + (pair - place * a.n_tiles)) * 4 + (warp >> 2);
                if (lane == 0) *to = slope_sum + (again ? *to : 0.f);
            }
            clear();
        }
    }
    if (lane == 0) tc::tma_store_wait_all();
}

template <class F>
__device__ __forceinline__ void pair_body(const LayerArgs& a) {
    static_assert(F::DYNAMIC_BYTES + sizeof(PairShared) <= SMEM_MOST && F::STAGES <= MAX_STAGES, "shared memory of a block");
    extern __shared__ uint8_t raw[];
    __shared__ PairShared sh;
    uint8_t* const ring_bytes = raw + ((1024u - (tc::smem_u32(raw) & 1023u)) & 1023u);
    uint8_t* const held_bytes = ring_bytes + F::RING_BYTES;
    const uint32_t ring = tc::smem_u32(ring_bytes), held = ring + F::RING_BYTES, slabs = held + F::HELD_BYTES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x >= 32 && threadIdx.x < 64) {
        tc::mbar_init(&sh.side[threadIdx.x >> 1 & 15][threadIdx.x & 1], 1);
        tc::fence_barrier_init();
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < F::STAGES; ++s) {
            tc::mbar_init(&sh.full[s], 1);
            tc::mbar_init(&sh.empty[s], 1);
        }
        for (int b = 0; b < 4; ++b) {
            tc::mbar_init(&sh.acc_full[b], 1);
            tc::mbar_init(&sh.acc_empty[b], 2 * F::DRAIN_WARPS);  // the first block counts the warps of both
        }
        tc::mbar_init(&sh.held_full, 1);
        tc::mbar_init(&sh.held_empty, 1);
        sh.abort = 0;
        tc::fence_barrier_init();
    }
    if (warp == F::DRAIN_WARPS) {
        tc::tmem_alloc_pair(&sh.tmem_base, 512);
        tc::tmem_relinquish_pair();
    }
    wait_for_kernel_before();
    lay_out<FORWARD, F::THREADS, BK>(a, sh);
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();  // both blocks' barriers and tensor memory exist before either is signalled
    tc::tc_fence_after_sync();
    const int rank = (int)tc::cluster_rank();
    if (warp < F::DRAIN_WARPS) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PAIR_DRAIN_REGISTERS));
        auto drain = [&](auto narrow) {
            with_activation<F::GRADIENT>(a, [&](auto act, auto beside) { pair_drain<F, decltype(act)::value, decltype(beside)::value, decltype(narrow)::value>(a, sh, slabs, rank); });
        };
        if constexpr (F::GATED && F::GRADIENT) drain(std::false_type());
        else if (Turns::of_pairs(F::GATED, F::GRADIENT, a.half).groups > 1) drain(std::true_type());
        else drain(std::false_type());
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PAIR_OTHER_REGISTERS));
        if (warp == F::DRAIN_WARPS && rank == 0) pair_multiplier<F>(a, sh, ring, held);
        if (warp == F::DRAIN_WARPS + 1 && lane == 0) pair_producer<F>(a, sh, ring_bytes, held_bytes, rank);
    }
    __syncwarp();
    if (*reinterpret_cast<volatile int*>(&sh.abort)) __nanosleep(1000000);  // a wait ran out: copies and MMAs under way land before the block ends
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();  // neither block leaves while the other may still signal it or read its operands
    if (warp == F::DRAIN_WARPS) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc_pair(sh.tmem_base, 512);
    }
}

template <class T, bool GATED, bool GRADIENT, bool RESIDENT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairForm<T, GATED, GRADIENT, RESIDENT>::THREADS, 1) layer_pairs_kernel(const __grid_constant__ LayerArgs a) {
    pair_body<PairForm<T, GATED, GRADIENT, RESIDENT>>(a);
}

template <class T, bool GATED, bool GRADIENT, bool RESIDENT>
int32_t launch_pairs_form(rtma_ctx* ctx, const LayerArgs& a, unsigned grid, bool& configured, cudaStream_t stream) {
    typedef PairForm<T, GATED, GRADIENT, RESIDENT> F;
    void (*kernel)(LayerArgs) = layer_pairs_kernel<T, GATED, GRADIENT, RESIDENT>;
    if (!configured) {
        RTMA_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, F::DYNAMIC_BYTES));
        configured = true;
    }
    launch_kernel(kernel, grid, F::THREADS, F::DYNAMIC_BYTES, stream, a);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

template <class T, bool GATED, bool RESIDENT>
int32_t launch_pairs(rtma_ctx* ctx, const LayerArgs& a, bool gradient, unsigned grid, cudaStream_t stream) {
    bool* once = ctx->layer_configured + (std::is_same<T, __half>::value ? 8 : 0) + (GATED ? 4 : 0) + (RESIDENT ? 2 : 0);
    return gradient ? launch_pairs_form<T, GATED, true, RESIDENT>(ctx, a, grid, once[1], stream) : launch_pairs_form<T, GATED, false, RESIDENT>(ctx, a, grid, once[0], stream);
}

}  // namespace
