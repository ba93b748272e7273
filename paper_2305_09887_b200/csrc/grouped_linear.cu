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

#include "grouped_linear.cuh"

RTMA_BOUNDS_TU()

namespace {

using namespace grouped;

enum Loading { COPIES, BULK, PAIR };

constexpr int BM = 128, BK = 64;
// Registers a thread.  COPIES is launched with 72 in the weight gradient (28 warps), otherwise with 80 (24 warps); the multiplier's
// four warps and the loading ones give some up to those that drain: 256 x 104 + 512 x 64 + 128 x 40 = 64,512 = 896 x 72, and with
// 384 loading threads 56,320 of 768 x 80.
constexpr int DRAIN_REGISTERS = 104, LOAD_REGISTERS = 64, MULTIPLY_REGISTERS = 40;
constexpr int SLAB_BYTES = 32 * 128;       // 32 rows of 64 16-bit values
constexpr int DW_WAVES = 2;                // tiles of a weight gradient for every block that runs at a time
constexpr int BIAS_ROWS = 1;               // of a slot: column sums of dY

template <class T, int MODE, int LOADING>
struct Form {
    static constexpr int BN = MODE == WEIGHT_GRADIENT ? 128 : 256;                                // widest tile
    static constexpr bool PAIRED = LOADING == PAIR;
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128 / (PAIRED ? 2 : 1);               // in one block
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    // the results of a tile leave while the next is drained, which is worth more than another stage
    static constexpr int RING_BYTES = (MODE == WEIGHT_GRADIENT ? 160 : 144) * 1024;
    static constexpr int STAGES = RING_BYTES / STAGE_BYTES;
    static constexpr int DRAIN_WARPS = 8;
    static constexpr int OUT_SLABS = MODE == WEIGHT_GRADIENT ? 2 : 4;                  // of a drain warp: 32 rows of 64 bytes on their way out
    static constexpr int OUT_BYTES = OUT_SLABS * 32 * 64;
    static constexpr int ACC_STAGES = MODE == WEIGHT_GRADIENT ? 2 : 1 << 20;           // after so many the accumulator is drained (or at a tile's end)
    static constexpr int ACC_COLUMNS = 256;                                            // dw: 128 of the product, 128 of the column sums
    static constexpr int ONES_BYTES = MODE == WEIGHT_GRADIENT ? 1024 : 0;
    static constexpr int DYNAMIC_BYTES = RING_BYTES + 1024 + DRAIN_WARPS * OUT_BYTES + ONES_BYTES;
    static constexpr bool A_ACROSS = MODE == WEIGHT_GRADIENT, B_ACROSS = MODE != INPUT_GRADIENT;  // MN-major
    // Of four warps that do nothing else.  Not more than stages: a group could be two rounds of the ring ahead of the multiplier, where
    // the parity of a barrier's phase says nothing.
    static constexpr int LOAD_GROUPS = LOADING != COPIES ? 0 : STAGES < 4 ? STAGES : 4;
    static constexpr int LOAD_WARPS = 4 * LOAD_GROUPS;
    using Walks = Walk<MODE, BM, BK, PAIRED>;
    static constexpr int THREADS = 32 * (DRAIN_WARPS + LOAD_WARPS + 4);
};

// Where the eight values of slab i that a loading thread (row 0..31 of the slab, unit 0..7 of the row) brings come from, and how
// many of them exist.
template <class T, int MODE>
__device__ __forceinline__ const T* source_a(const LinearArgs& a, const Walk<MODE, BM, BK>& w, int i, int row, int unit, int& valid) {
    const T* A = static_cast<const T*>(a.A);
    if constexpr (MODE == WEIGHT_GRADIENT) {
        const int k = w.k0 + 32 * (i & 1) + row, c = w.m0 + 64 * (i >> 1) + 8 * unit;
        valid = k < w.k_end ? max(0, min(8, a.d_in - c)) : 0;
        return valid ? A + (w.row0 + k) * a.lda + c : A;
    } else {
        const int r = 32 * i + row, c = w.k0 + 8 * unit;
        valid = r < w.rows ? max(0, min(8, w.k_end - c)) : 0;
        return valid ? A + (w.row0 + r) * a.lda + c : A;
    }
}
template <class T, int MODE>
__device__ __forceinline__ const T* source_b(const LinearArgs& a, const Walk<MODE, BM, BK>& w, int i, int row, int unit, int& valid) {
    const T* B = static_cast<const T*>(a.B);
    if constexpr (MODE == INPUT_GRADIENT) {
        const int r = w.n0 + 32 * i + row, c = w.k0 + 8 * unit;
        valid = r < a.d_in ? max(0, min(8, w.k_end - c)) : 0;
        return valid ? B + w.part * a.w_stride + r * a.ldb + c : B;
    } else {
        const int k = w.k0 + 32 * (i & 1) + row, c = w.n0 + 64 * (i >> 1) + 8 * unit;
        valid = k < w.k_end ? max(0, min(8, a.d_out - c)) : 0;
        if constexpr (MODE == WEIGHT_GRADIENT) return valid ? B + (w.row0 + k) * a.ldb + c : B;
        else return valid ? B + w.part * a.w_stride + k * a.ldb + c : B;
    }
}

template <int SIZE>
__device__ __forceinline__ void copy(uint32_t dst, const void* src, int bytes) {  // the rest of the SIZE bytes becomes zero
    if constexpr (SIZE == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(bytes), "n"(SIZE) : "memory");
}
// 16 bytes of which `bytes` exist, from a multiple of SIZE
template <int SIZE>
__device__ __forceinline__ void copy_pieces(uint32_t dst, const void* src, int bytes) {
#pragma unroll
    for (int i = 0; i < 16 / SIZE; ++i) {
        const int here = max(0, min(SIZE, bytes - i * SIZE));
        copy<SIZE>(dst + i * SIZE, here ? static_cast<const char*>(src) + i * SIZE : src, here);
    }
}
// this thread's copies have landed and the tensor cores may read them
__device__ __forceinline__ void copies_done() {
    asm volatile("cp.async.wait_all;" ::: "memory");
    tc::fence_proxy_async_smem();
}

// What one thread brings of an operand (rows 0..15 and 16 more, unit 0..7 of every slab): an address, steps from there.
template <class T, int MODE, bool IS_B>
struct Source {
    static constexpr bool ACROSS = IS_B ? MODE != INPUT_GRADIENT : MODE == WEIGHT_GRADIENT;
    const T* p;      // the tile's first
    int near, cols;  // along: rows from this thread's on, terms;  across: terms from this thread's row on, columns from its unit on
    int64_t half;    // elements between 16 rows
    __device__ __forceinline__ void open(const LinearArgs& a, const Walk<MODE, BM, BK>& w, int row, int unit) {
        const T* base = static_cast<const T*>(IS_B ? a.B : a.A);
        const int64_t ld = IS_B ? a.ldb : a.lda;
        half = 16 * ld;
        if constexpr (ACROSS) {
            const int c = (IS_B ? w.n0 : w.m0) + 8 * unit;
            near = w.k_end - row;
            cols = (IS_B ? a.d_out : a.d_in) - c;
            p = base + (MODE == WEIGHT_GRADIENT ? (w.row0 + row) * ld : w.part * a.w_stride + row * ld) + c;
        } else {
            near = (IS_B ? a.d_in - w.n0 : w.rows) - row;
            cols = w.k_end - 8 * unit;
            p = base + (IS_B ? w.part * a.w_stride + (w.n0 + row) * ld : (w.row0 + row) * ld) + 8 * unit;
        }
    }
    // half h of slab i of the stage that starts with term k0; valid: how many of the eight exist (the tile's first address if none does)
    __device__ __forceinline__ const T* at(int i, int h, int k0, int& valid) const {
        if constexpr (ACROSS) {
            const int k = k0 + 32 * (i & 1) + 16 * h, c = 64 * (i >> 1);
            valid = k < near ? max(0, min(8, cols - c)) : 0;
            return valid ? p + (k >> 4) * half + c : p;
        } else {
            valid = 32 * i + 16 * h < near ? max(0, min(8, cols - k0)) : 0;
            return valid ? p + (2 * i + h) * half + k0 : p;
        }
    }
};

// `slabs` slabs of an operand into a stage, by 128 threads (t).
template <class T, int MODE, bool IS_B>
__device__ __forceinline__ void copy_operand(const LinearArgs& a, const Walk<MODE, BM, BK>& w, uint32_t to, int slabs, int granule, int t) {
    const int row = t >> 3, unit = t & 7;
    Source<T, MODE, IS_B> from;
    from.open(a, w, row, unit);
    to += row * 128 + ((unit ^ (row & 7)) << 4);  // (16 rows do not change row mod 8)
#pragma unroll 2
    for (int i = 0; i < slabs; ++i, to += SLAB_BYTES) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int valid;
            const T* p = from.at(i, h, w.k0, valid);
            const uint32_t dst = to + h * (SLAB_BYTES / 2);
            if (granule >= 16) copy_pieces<16>(dst, p, valid * (int)sizeof(T));
            else if (granule == 8) copy_pieces<8>(dst, p, valid * (int)sizeof(T));
            else if (granule == 4) copy_pieces<4>(dst, p, valid * (int)sizeof(T));
            else {
                Eight<T> e;
                e.load(p, valid, granule);
                store_16(dst, e.w[0]);
            }
        }
    }
}

// The bulk-tensor loads of a stage's operand, by one thread.
template <class T, int MODE, int LOADING>
__device__ __forceinline__ uint32_t bulk_bytes_b(const LinearArgs& a) {
    return Form<T, MODE, LOADING>::B_ACROSS ? (uint32_t)((a.BN + 63) / 64) * 2 * SLAB_BYTES : (uint32_t)a.BN * 128u;
}
template <int MODE>
__device__ __forceinline__ void bulk_a(const LinearArgs& a, const Walk<MODE, BM, BK>& w, uint8_t* to, uint64_t* bar) {
    if constexpr (MODE == WEIGHT_GRADIENT) {
        for (int i = 0; i < 2; ++i) tc::tma_load_3d(to + 2 * i * SLAB_BYTES, &a.map_a, bar, w.m0 + 64 * i, (int)w.row0 + w.k0, 0);
    } else {
        tc::tma_load_3d(to, &a.map_a, bar, w.k0, (int)w.row0, 0);
    }
}
template <int MODE>
__device__ __forceinline__ void bulk_b(const LinearArgs& a, const Walk<MODE, BM, BK>& w, uint8_t* to, uint64_t* bar) {
    const int z = MODE != WEIGHT_GRADIENT && a.w_stride ? w.part : 0;
    if constexpr (MODE == INPUT_GRADIENT) {
        tc::tma_load_3d(to, &a.map_b, bar, w.k0, w.n0, z);
    } else {
        const int r = MODE == FORWARD ? w.k0 : (int)w.row0 + w.k0;
        for (int i = 0; 64 * i < a.BN; ++i) tc::tma_load_3d(to + 2 * i * SLAB_BYTES, &a.map_b, bar, w.n0 + 64 * i, r, z);
    }
}

// Stages by copies, which groups of four warps fill in turn.  A group waits for its own copies and makes them visible to the tensor
// cores itself: a fence in the multiplier's warp waits for everything that the block has on its way, which made a stage of
// the weight gradient of 1M x 256 x 47 in fp16 cost 2700 cycles (375 us; with groups 256 us).  An operand whose rows do lie on 16-byte
// boundaries still comes in bulk.
template <class T, int MODE>
__device__ __forceinline__ void copy_role(const LinearArgs& a, Shared& sh, uint8_t* ring, int t, int group) {
    typedef Form<T, MODE, COPIES> F;
    const int slabs = F::B_ACROSS ? 2 * ((a.BN + 63) / 64) : (a.BN + 31) / 32;
    Walk<MODE, BM, BK> w;
    tc::RingAt at;
    int turn = 0;
    for (bool more = w.first(a, sh); more; more = w.next(a, sh), at.advance(F::STAGES)) {
        const bool mine = turn == group;
        turn = turn + 1 == F::LOAD_GROUPS ? 0 : turn + 1;
        if (!mine) continue;
        if (!wait_for(&sh.empty[at.s], at.phase ^ 1u, sh, a.error_word)) break;
        uint8_t* stage = ring + at.s * F::STAGE_BYTES;
        uint64_t* bar = &sh.full[at.s];
        const bool cut = MODE == WEIGHT_GRADIENT && w.k0 + BK > w.k_end;  // rows of the next part must not be summed
        const bool a_whole = a.in_bulk & 1 && !cut, b_whole = a.in_bulk & 2 && !cut;
        if (t == 0 && (a_whole || b_whole)) {  // (announced before this warp's arrival)
            tc::mbar_expect_tx(bar, (a_whole ? F::A_BYTES : 0u) + (b_whole ? bulk_bytes_b<T, MODE, COPIES>(a) : 0u));
            if (a_whole) bulk_a<MODE>(a, w, stage, bar);
            if (b_whole) bulk_b<MODE>(a, w, stage + F::A_BYTES, bar);
        }
        if (!a_whole) copy_operand<T, MODE, false>(a, w, tc::smem_u32(stage), 4, a.va, t);
        if (!b_whole) copy_operand<T, MODE, true>(a, w, tc::smem_u32(stage) + F::A_BYTES, slabs, a.vb, t);
        copies_done();
        __syncwarp();
        if ((t & 31) == 0) tc::mbar_arrive(bar);
    }
}

// One warp with bulk-tensor loads.  Rows behind the end of a tile belong to the next part: they only reach results that are not
// written, but in the weight gradient they would be summed, so the last rows of a part are copied by the warp's lanes, with zeros
// behind them.
template <class T, int MODE>
__device__ __forceinline__ void bulk_role(const LinearArgs& a, Shared& sh, uint8_t* ring, int lane) {
    typedef Form<T, MODE, BULK> F;
    const uint32_t b_bytes = bulk_bytes_b<T, MODE, BULK>(a);
    if (lane == 0) {
        tc::prefetch_tensormap(&a.map_a);
        tc::prefetch_tensormap(&a.map_b);
    }
    Walk<MODE, BM, BK> w;
    tc::RingAt at;
    for (bool more = w.first(a, sh); more; more = w.next(a, sh), at.advance(F::STAGES)) {
        if (!wait_for(&sh.empty[at.s], at.phase ^ 1u, sh, a.error_word)) return;
        uint8_t* stage = ring + at.s * F::STAGE_BYTES;
        uint64_t* bar = &sh.full[at.s];
        if (MODE == WEIGHT_GRADIENT && w.k0 + BK > w.k_end) {
            const int slabs = 2 * ((a.BN + 63) / 64);
            for (int j = lane; j < (4 + slabs) * 256; j += 32) {
                const int i = j >> 8, row = (j >> 3) & 31, unit = j & 7;
                int valid;
                const T* p = i < 4 ? source_a<T, MODE>(a, w, i, row, unit, valid) : source_b<T, MODE>(a, w, i - 4, row, unit, valid);
                copy<16>(tc::smem_u32(stage) + i * SLAB_BYTES + row * 128 + ((unit ^ (row & 7)) << 4), p, valid * (int)sizeof(T));
            }
            copies_done();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar);
        } else if (lane == 0) {
            tc::mbar_arrive_expect_tx(bar, F::A_BYTES + b_bytes);
            bulk_a<MODE>(a, w, stage, bar);
            bulk_b<MODE>(a, w, stage + F::A_BYTES, bar);
        }
        __syncwarp();
    }
}

// A pair of blocks: each loads its own rows and its half of the right operand's columns, announced and counted on the first block's
// barrier (the other's bytes may land before the announcement: the phase still lacks its arrival).
template <class T, int MODE>
__device__ __forceinline__ void pair_role(const LinearArgs& a, Shared& sh, uint8_t* ring, int rank) {
    typedef Form<T, MODE, PAIR> F;
    tc::prefetch_tensormap(&a.map_a);
    tc::prefetch_tensormap(&a.map_b);
    typename F::Walks w;
    tc::RingAt at;
    int filled = 0;  // stages, F::STAGES at most
    bool ok = true;
    for (bool more = w.first(a, sh); more; more = w.next(a, sh), at.advance(F::STAGES)) {
        if (!wait_for<true>(&sh.empty[at.s], at.phase ^ 1u, sh, a.error_word)) {
            ok = false;
            break;
        }
        filled = min(filled + 1, F::STAGES);
        uint8_t* stage = ring + at.s * F::STAGE_BYTES;
        if (rank == 0) tc::mbar_arrive_expect_tx(&sh.full[at.s], 2 * F::STAGE_BYTES);
        const uint32_t bar = tc::leader_addr(&sh.full[at.s]);
        const int z = a.w_stride ? w.part : 0, n0 = w.n0 + rank * (F::BN / 2);
        tc::tma_load_3d_pair(stage, &a.map_a, bar, w.k0, (int)w.row0, 0);
        if constexpr (MODE == FORWARD) {
            for (int i = 0; i < 2; ++i) tc::tma_load_3d_pair(stage + F::A_BYTES + 2 * i * SLAB_BYTES, &a.map_b, bar, n0 + 64 * i, w.k0, z);
        } else {
            tc::tma_load_3d_pair(stage + F::A_BYTES, &a.map_b, bar, w.k0, n0, z);
        }
    }
    // No signal stays under way: every stage filled is waited for until both blocks have it back or, after a give-up, until its loads
    // have landed (the first block, for both).
    for (int n = 0; n < filled; ++n) {
        // the oldest first: `filled` stages back, of the round before where that is behind the ring's start
        const int back = filled - n, s = (at.s - back + F::STAGES) % F::STAGES;
        const uint32_t parity = s < at.s ? at.phase : at.phase ^ 1u;
        if (!ok || !wait_for<true>(&sh.empty[s], parity, sh, a.error_word)) {
            ok = false;
            if (rank == 0)
                for (uint32_t i = 0; i < (1u << 14) && !tc::mbar_try_wait_cluster(&sh.full[s], parity); ++i) {}
        }
    }
}

// A stage's MMAs, by one warp.
template <class T, int MODE, int LOADING>
__device__ __forceinline__ void multiply_stage(const LinearArgs& a, uint32_t d, uint32_t stage, int terms, uint32_t accumulate, uint32_t ones) {
    typedef Form<T, MODE, LOADING> F;
    const uint32_t format = std::is_same<T, __half>::value ? 0u : 1u;  // fp16 or bf16 operands, fp32 sums
    const uint32_t idesc = (1u << 4) | (format << 7) | (format << 10) | ((F::A_ACROSS ? 1u : 0u) << 15) | ((F::B_ACROSS ? 1u : 0u) << 16) |
                           ((uint32_t)(a.BN >> 3) << 17) | ((uint32_t)((F::PAIRED ? 2 * BM : BM) >> 4) << 24);
    const uint64_t desc = tc::smem_desc_sw128(0, 2 * SLAB_BYTES, 1024);  // atoms of 64 columns lie two slabs apart
    constexpr uint32_t a_step = F::A_ACROSS ? 128 : 2, b_step = F::B_ACROSS ? 128 : 2;  // 16 terms further, in units of 16 bytes
    constexpr uint32_t a_plane = F::A_BYTES >> 4;
    const uint64_t da = desc + (stage >> 4), db = da + a_plane;
    const int steps = (terms + 15) >> 4;
#pragma unroll
    for (int k = 0; k < BK / 16; ++k)
        if (k < steps) {
            if constexpr (F::PAIRED) tc::mma_pair_by_warp(d, da + k * a_step, db + k * b_step, idesc, k ? 1u : accumulate);
            else tc::mma_by_warp(d, da + k * a_step, db + k * b_step, idesc, k ? 1u : accumulate);
        }
    if (MODE == WEIGHT_GRADIENT && ones) {  // 128 rows of ones, all from the same 1024 bytes
        const uint64_t one = tc::smem_desc_sw128(ones, 0, 0);
#pragma unroll
        for (int k = 0; k < BK / 16; ++k)
            if (k < steps) tc::mma_by_warp(d + 128, one, db + k * b_step, idesc, k ? 1u : accumulate);
    }
}

template <class T, int MODE, int LOADING>
__device__ __forceinline__ void multiply_role(const LinearArgs& a, Shared& sh, uint32_t ring, uint32_t ones) {
    typedef Form<T, MODE, LOADING> F;
    typename F::Walks w;
    tc::RingAt at, acc;
    int held = 0;  // stages in the accumulator
    auto commit = [](uint64_t* bar) {
        if constexpr (F::PAIRED) tc::commit_pair_by_warp(bar);
        else tc::commit_by_warp(bar);
    };
    for (bool more = w.first(a, sh); more; more = w.next(a, sh)) {
        if (held == 0 && !wait_for<F::PAIRED>(&sh.acc_empty[acc.s], acc.phase ^ 1u, sh, a.error_word)) return;
        if (!wait_for<F::PAIRED>(&sh.full[at.s], at.phase, sh, a.error_word)) return;
        tc::tc_fence_after_sync();
        __syncwarp();
        multiply_stage<T, MODE, LOADING>(a, sh.tmem_base + acc.s * F::ACC_COLUMNS, ring + at.s * F::STAGE_BYTES, min(BK, w.k_end - w.k0), held ? 1u : 0u,
                                         a.db && w.m0 == 0 ? ones : 0u);
        commit(&sh.empty[at.s]);
        at.advance(F::STAGES);
        if (++held == F::ACC_STAGES || w.last_stage()) {
            held = 0;
            commit(&sh.acc_full[acc.s]);
            acc.advance(2);
        }
    }
}

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
__device__ __forceinline__ void linear_body(const LinearArgs& a) {
    typedef Form<T, MODE, LOADING> F;
    static_assert(F::DYNAMIC_BYTES + sizeof(Shared) <= SMEM_MOST && F::STAGES <= MAX_STAGES, "shared memory of a block");
    extern __shared__ uint8_t raw[];
    __shared__ Shared sh;
    uint8_t* ring_bytes = raw + ((1024u - (tc::smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t ring = tc::smem_u32(ring_bytes), slabs = ring + F::RING_BYTES, ones = slabs + F::DRAIN_WARPS * F::OUT_BYTES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int MULTIPLIER = F::DRAIN_WARPS + F::LOAD_WARPS;
    if (threadIdx.x == 0) {
        for (int s = 0; s < F::STAGES; ++s) {
            tc::mbar_init(&sh.full[s], LOADING == COPIES ? 4 : 1);
            tc::mbar_init(&sh.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc::mbar_init(&sh.acc_full[b], 1);
            tc::mbar_init(&sh.acc_empty[b], (F::PAIRED ? 2 : 1) * F::DRAIN_WARPS);  // a pair's first block counts the warps of both
        }
        sh.abort = 0;
        tc::fence_barrier_init();
    }
    if (warp == MULTIPLIER) {
        if constexpr (F::PAIRED) {
            tc::tmem_alloc_pair(&sh.tmem_base, 2 * F::ACC_COLUMNS);
            tc::tmem_relinquish_pair();
        } else {
            tc::tmem_alloc(&sh.tmem_base, 2 * F::ACC_COLUMNS);
            tc::tmem_relinquish();
        }
    }
    if (MODE == WEIGHT_GRADIENT && threadIdx.x < 64) {
        const uint32_t one = std::is_same<T, __half>::value ? 0x3C003C00u : 0x3F803F80u;
        store_16(ones + 16 * threadIdx.x, make_uint4(one, one, one, one));
        tc::fence_proxy_async_smem();
    }
    wait_for_kernel_before();
    lay_out<MODE, F::THREADS, BK>(a, sh);
    tc::tc_fence_before_sync();
    __syncthreads();
    if constexpr (F::PAIRED) tc::cluster_sync();  // both blocks' barriers and tensor memory exist before either is signalled
    tc::tc_fence_after_sync();
    const int rank = F::PAIRED ? (int)tc::cluster_rank() : 0;
    if (warp < F::DRAIN_WARPS) {
        if constexpr (LOADING == COPIES) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(DRAIN_REGISTERS));
        drain_role<T, MODE, LOADING>(a, sh, slabs);
    } else if (warp < MULTIPLIER) {
        if constexpr (LOADING == COPIES) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LOAD_REGISTERS));
            const int t = threadIdx.x - 32 * F::DRAIN_WARPS;
            copy_role<T, MODE>(a, sh, ring_bytes, t & 127, t >> 7);
        }
    } else {
        if constexpr (LOADING == COPIES) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(MULTIPLY_REGISTERS));
        if (warp == MULTIPLIER && rank == 0) multiply_role<T, MODE, LOADING>(a, sh, ring, ones);
        if constexpr (LOADING == BULK)
            if (warp == MULTIPLIER + 1) bulk_role<T, MODE>(a, sh, ring_bytes, lane);
        if constexpr (F::PAIRED)
            if (warp == MULTIPLIER + 1 && lane == 0) pair_role<T, MODE>(a, sh, ring_bytes, rank);
    }
    __syncwarp();
    if (*reinterpret_cast<volatile int*>(&sh.abort)) __nanosleep(1000000);  // a wait ran out: copies and MMAs under way land before the block ends
    tc::tc_fence_before_sync();
    __syncthreads();
    if constexpr (F::PAIRED) tc::cluster_sync();  // neither block leaves while the other may still signal it or read its operands
    if (warp == MULTIPLIER) {
        tc::tc_fence_after_sync();
        if constexpr (F::PAIRED) tc::tmem_dealloc_pair(sh.tmem_base, 2 * F::ACC_COLUMNS);
        else tc::tmem_dealloc(sh.tmem_base, 2 * F::ACC_COLUMNS);
    }
}

template <class T, int MODE, int LOADING>
__global__ void __launch_bounds__(Form<T, MODE, LOADING>::THREADS, 1) linear_kernel(const __grid_constant__ LinearArgs a) {
    linear_body<T, MODE, LOADING>(a);
}
template <class T, int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Form<T, MODE, PAIR>::THREADS, 1) linear_pair_kernel(const __grid_constant__ LinearArgs a) {
    linear_body<T, MODE, PAIR>(a);
}

// The slots of every part added up in order.  A block takes 128 neighbouring places of a slot, its warps every eighth slot each; the
// row behind the weights is the bias's, whose partial sums lie in bias_rows rows (added up one after the other by one thread each they
// took 414 us for 16 parts; so, the kernel takes 10).
constexpr int REDUCE_THREADS = 256;
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
    float* to = row < a.d_in ? a.dW + part * a.dw_stride + (int64_t)row * a.d_out + col : a.db + part * a.db_stride + col;
    if (col < a.d_out) to[0] = s.x;
    if (col + 1 < a.d_out) to[1] = s.y;
    if (col + 2 < a.d_out) to[2] = s.z;
    if (col + 3 < a.d_out) to[3] = s.w;
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

int32_t run_rows(rtma_ctx* ctx, const char* who, bool transposed, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                 const void* A, int64_t lda, const void* W, int64_t w_stride, const void* b, int64_t b_stride, void* out, int64_t ldo, void* stream_) {
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_linear(ctx, who, dtype, n, G, offsets, d_in, d_out));
    if (n == 0) return RTMA_OK;
    if (!A || !W || !out) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: null pointer", who);
    const int K = transposed ? d_out : d_in, N = transposed ? d_in : d_out;
    if (lda < K || ldo < N) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: rows of %d and %d values lie closer than that", who, K, N);
    if (A == out) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: the result must not overlap the rows", who);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
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
    RTMA_TRY(prepare_row_call(ctx, dtype == RTMA_F32 ? split_planes_bytes(a) : pad ? padded : 0, stream));
    if (pad) RTMA_TRY(pad_matrices(ctx, a, stream));
    return transposed ? launch_linear<INPUT_GRADIENT>(ctx, dtype, a, KC_GEMM_DGRAD, stream) : launch_linear<FORWARD>(ctx, dtype, a, KC_GEMM_FWD, stream);
}

}  // namespace

extern "C" int32_t rtma_grouped_linear(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                                       const void* X, int64_t ldx, const void* W, int64_t w_stride, const void* b, int64_t b_stride, void* Y,
                                       int64_t ldy, void* stream) {
    return run_rows(ctx, "rtma_grouped_linear", false, dtype, n, G, offsets, d_in, d_out, X, ldx, W, w_stride, b, b_stride, Y, ldy, stream);
}

extern "C" int32_t rtma_grouped_linear_dx(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                                          const void* dY, int64_t lddy, const void* W, int64_t w_stride, void* dX, int64_t lddx, void* stream) {
    return run_rows(ctx, "rtma_grouped_linear_dx", true, dtype, n, G, offsets, d_in, d_out, dY, lddy, W, w_stride, nullptr, 0, dX, lddx, stream);
}

extern "C" int32_t rtma_grouped_linear_dw(rtma_ctx* ctx, int32_t dtype, int64_t n, int32_t G, const int64_t* offsets, int32_t d_in, int32_t d_out,
                                          const void* X, int64_t ldx, const void* dY, int64_t lddy, float* dW, int64_t dw_stride, float* db,
                                          int64_t db_stride, void* stream_) {
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_linear(ctx, "rtma_grouped_linear_dw", dtype, n, G, offsets, d_in, d_out));
    if (!dW || (n > 0 && (!X || !dY))) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_grouped_linear_dw: null pointer");
    if (ldx < d_in || lddy < d_out) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_grouped_linear_dw: rows of %d and %d values lie closer than that", d_in, d_out);
    const int64_t weights = (int64_t)d_in * d_out;
    const bool shared = G > 1 && dw_stride == 0;
    if (G > 1 && db && (db_stride == 0) != shared)
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_grouped_linear_dw: either both gradients are one for all parts or neither");
    if (G > 1 && !shared && ((dw_stride < weights && dw_stride > -weights) || (db && db_stride < d_out && db_stride > -d_out)))
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_grouped_linear_dw: gradients of the parts overlap");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
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
    a.ldo = ceil_div(d_out, 8) * 8;
    a.go = 32;
    const int64_t slot_rows = a.tiles * (d_in + a.bias_rows);
    RTMA_TRY(prepare_row_call(ctx, 256 + sizeof(float) * slot_rows * a.ldo, stream));
    a.chunk_rows = reinterpret_cast<int32_t*>(ctx->arena);
    a.out = ctx->arena + 256;
    a.vo = dtype != RTMA_F32 && slot_rows < (int64_t(1) << 31) && make_store_map(&a.map_o, RTMA_F32, a.out, slot_rows, a.ldo, a.ldo);
    if (n > 0) RTMA_TRY(launch_linear<WEIGHT_GRADIENT>(ctx, dtype, a, KC_GEMM_WGRAD, stream));
    {
        KernelScope ks(ctx, KC_REDUCE_SGD, stream);
        launch_kernel(linear_reduce_kernel, dim3((unsigned)ceil_div((d_in + 1) * a.ldo, 128), (unsigned)a.G), REDUCE_THREADS, 0, stream, a);
    }
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}
