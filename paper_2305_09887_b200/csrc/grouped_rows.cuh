// The kernel of the products of 16-bit rows with the matrices of their parts, without the way of its results out: how operands are
// staged, by copies or bulk-tensor loads, the MMAs, and the block that runs these roles.  A kernel adds what its drain warps do with the
// accumulators.
//
// GATED (forward walks): the matrix is two of equal width side by side, `up` columns apart, and a tile has the same BN columns (128 at
// most) of both: the left one's at column 0 of the accumulator, the right one's at column 128.
#pragma once

#include "grouped_linear.cuh"

#ifdef __CUDACC__

namespace grouped {

enum Loading { COPIES, BULK, PAIR };

constexpr int BM = 128, BK = 64;
// Registers a thread.  COPIES is launched with 72 in the weight gradient (28 warps), otherwise with 80 (24 warps); the multiplier's
// four warps and the loading ones give some up to those that drain: 256 x 104 + 512 x 64 + 128 x 40 = 64,512 = 896 x 72, and with
// 384 loading threads 56,320 of 768 x 80.
constexpr int DRAIN_REGISTERS = 104, LOAD_REGISTERS = 64, MULTIPLY_REGISTERS = 40;
constexpr int SLAB_BYTES = 32 * 128;       // 32 rows of 64 16-bit values

template <class T_, int MODE_, int LOADING_, bool GATED_ = false, int DRAIN_WARPS_ = 8>
struct Form {
    typedef T_ T;
    static constexpr int MODE = MODE_, LOADING = LOADING_;
    static constexpr bool GATED = GATED_;
    static_assert(!GATED || MODE == FORWARD, "a gated layer is walked forward");
    static constexpr int BN = MODE == WEIGHT_GRADIENT ? 128 : 256;                                // widest tile
    static constexpr bool PAIRED = LOADING == PAIR;
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128 / (PAIRED ? 2 : 1);               // in one block
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    // the results of a tile leave while the next is drained, which is worth more than another stage
    static constexpr int RING_BYTES = (MODE == WEIGHT_GRADIENT ? 160 : 144) * 1024;
    static constexpr int STAGES = RING_BYTES / STAGE_BYTES;
    static constexpr int DRAIN_WARPS = DRAIN_WARPS_;
    static constexpr int OUT_SLABS = MODE == WEIGHT_GRADIENT ? 2 : 32 / DRAIN_WARPS;   // of a drain warp: 32 rows of 64 bytes on their way out
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
    // Registers go over to the warps that drain: from those that copy, or (16 drain warps: 640 threads at 96, 512 x 104 + 128 x 64 = 640 x 96)
    // from the multiplier's four
    static constexpr bool MOVES = LOADING == COPIES || DRAIN_WARPS == 16;
    static constexpr int MULTIPLY = LOADING == COPIES ? MULTIPLY_REGISTERS : 64;
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
template <class F>
__device__ __forceinline__ uint32_t bulk_bytes_b(const LinearArgs& a) {
    return F::B_ACROSS ? (uint32_t)((a.BN + 63) / 64) * (F::GATED ? 4 : 2) * SLAB_BYTES : (uint32_t)a.BN * 128u;
}
template <int MODE>
__device__ __forceinline__ void bulk_a(const LinearArgs& a, const Walk<MODE, BM, BK>& w, uint8_t* to, uint64_t* bar) {
    if constexpr (MODE == WEIGHT_GRADIENT) {
        for (int i = 0; i < 2; ++i) tc::tma_load_3d(to + 2 * i * SLAB_BYTES, &a.map_a, bar, w.m0 + 64 * i, (int)w.row0 + w.k0, 0);
    } else {
        tc::tma_load_3d(to, &a.map_a, bar, w.k0, (int)w.row0, 0);
    }
}
template <class F>
__device__ __forceinline__ void bulk_b(const LinearArgs& a, const Walk<F::MODE, BM, BK>& w, uint8_t* to, uint64_t* bar) {
    constexpr int MODE = F::MODE;
    const int z = MODE != WEIGHT_GRADIENT && a.w_stride ? w.part : 0;
    if constexpr (MODE == INPUT_GRADIENT) {
        tc::tma_load_3d(to, &a.map_b, bar, w.k0, w.n0, z);
    } else {
        const int r = MODE == FORWARD ? w.k0 : (int)w.row0 + w.k0;
        for (int i = 0; 64 * i < a.BN; ++i) tc::tma_load_3d(to + 2 * i * SLAB_BYTES, &a.map_b, bar, w.n0 + 64 * i, r, z);
        if constexpr (F::GATED) {
            to += (a.BN + 63) / 64 * 2 * SLAB_BYTES;
            for (int i = 0; 64 * i < a.BN; ++i) tc::tma_load_3d(to + 2 * i * SLAB_BYTES, &a.map_b, bar, a.up + w.n0 + 64 * i, r, z);
        }
    }
}

// Stages by copies, which groups of four warps fill in turn.  A group waits for its own copies and makes them visible to the tensor
// cores itself: a fence in the multiplier's warp waits for everything that the block has on its way, which made a stage of
// the weight gradient of 1M x 256 x 47 in fp16 cost 2700 cycles (375 us; with groups 256 us).  An operand whose rows do lie on 16-byte
// boundaries still comes in bulk.
template <class F>
__device__ __forceinline__ void copy_role(const LinearArgs& a, Shared& sh, uint8_t* ring, int t, int group) {
    typedef typename F::T T;
    constexpr int MODE = F::MODE;
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
            tc::mbar_expect_tx(bar, (a_whole ? F::A_BYTES : 0u) + (b_whole ? bulk_bytes_b<F>(a) : 0u));
            if (a_whole) bulk_a<MODE>(a, w, stage, bar);
            if (b_whole) bulk_b<F>(a, w, stage + F::A_BYTES, bar);
        }
        if (!a_whole) copy_operand<T, MODE, false>(a, w, tc::smem_u32(stage), 4, a.va, t);
        if constexpr (!F::GATED)  // (two matrices always come in bulk)
            if (!b_whole) copy_operand<T, MODE, true>(a, w, tc::smem_u32(stage) + F::A_BYTES, slabs, a.vb, t);
        copies_done();
        __syncwarp();
        if ((t & 31) == 0) tc::mbar_arrive(bar);
    }
}

// One warp with bulk-tensor loads.  Rows behind the end of a tile belong to the next part: they only reach results that are not
// written, but in the weight gradient they would be summed, so the last rows of a part are copied by the warp's lanes, with zeros
// behind them.
template <class F>
__device__ __forceinline__ void bulk_role(const LinearArgs& a, Shared& sh, uint8_t* ring, int lane) {
    typedef typename F::T T;
    constexpr int MODE = F::MODE;
    const uint32_t b_bytes = bulk_bytes_b<F>(a);
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
            bulk_b<F>(a, w, stage + F::A_BYTES, bar);
        }
        __syncwarp();
    }
}

// A pair of blocks: each loads its own rows and its half of the right operand's columns, announced and counted on the first block's
// barrier (the other's bytes may land before the announcement: the phase still lacks its arrival).
template <class F>
__device__ __forceinline__ void pair_role(const LinearArgs& a, Shared& sh, uint8_t* ring, int rank) {
    constexpr int MODE = F::MODE;
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
        const int z = a.w_stride ? w.part : 0, n0 = w.n0 + rank * (F::GATED ? a.up : F::BN / 2);
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
template <class F>
__device__ __forceinline__ void multiply_stage(const LinearArgs& a, uint32_t d, uint32_t stage, int terms, uint32_t accumulate, uint32_t ones) {
    constexpr int MODE = F::MODE;
    const uint32_t format = std::is_same<typename F::T, __half>::value ? 0u : 1u;  // fp16 or bf16 operands, fp32 sums
    // two matrices: one MMA for both where their columns lie behind one another in shared and in tensor memory
    const bool both = F::GATED && (F::PAIRED || a.BN == 128);
    const uint32_t idesc = (1u << 4) | (format << 7) | (format << 10) | ((F::A_ACROSS ? 1u : 0u) << 15) | ((F::B_ACROSS ? 1u : 0u) << 16) |
                           ((uint32_t)((both ? 256 : a.BN) >> 3) << 17) | ((uint32_t)((F::PAIRED ? 2 * BM : BM) >> 4) << 24);
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
    if constexpr (F::GATED && !F::PAIRED) {
        if (!both) {
            const uint64_t right = db + (uint32_t)((a.BN + 63) / 64) * (2 * SLAB_BYTES >> 4);
#pragma unroll
            for (int k = 0; k < BK / 16; ++k)
                if (k < steps) tc::mma_by_warp(d + 128, da + k * a_step, right + k * b_step, idesc, k ? 1u : accumulate);
        }
    }
    if (MODE == WEIGHT_GRADIENT && ones) {  // 128 rows of ones, all from the same 1024 bytes
        const uint64_t one = tc::smem_desc_sw128(ones, 0, 0);
#pragma unroll
        for (int k = 0; k < BK / 16; ++k)
            if (k < steps) tc::mma_by_warp(d + 128, one, db + k * b_step, idesc, k ? 1u : accumulate);
    }
}

template <class F>
__device__ __forceinline__ void multiply_role(const LinearArgs& a, Shared& sh, uint32_t ring, uint32_t ones) {
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
        multiply_stage<F>(a, sh.tmem_base + acc.s * F::ACC_COLUMNS, ring + at.s * F::STAGE_BYTES, min(BK, w.k_end - w.k0), held ? 1u : 0u,
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

// drain: what a drain warp does, with the shared memory address of the slabs
template <class F, class S, class Drain>
__device__ __forceinline__ void linear_body(const LinearArgs& a, S& sh, Drain drain) {
    typedef typename F::T T;
    constexpr int MODE = F::MODE, LOADING = F::LOADING;
    static_assert(F::DYNAMIC_BYTES + sizeof(S) <= SMEM_MOST && F::STAGES <= MAX_STAGES, "shared memory of a block");
    extern __shared__ uint8_t raw[];
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
        if constexpr (F::MOVES) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(DRAIN_REGISTERS));
        drain(slabs);
    } else if (warp < MULTIPLIER) {
        if constexpr (LOADING == COPIES) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LOAD_REGISTERS));
            const int t = threadIdx.x - 32 * F::DRAIN_WARPS;
            copy_role<F>(a, sh, ring_bytes, t & 127, t >> 7);
        }
    } else {
        if constexpr (F::MOVES) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F::MULTIPLY));
        if (warp == MULTIPLIER && rank == 0) multiply_role<F>(a, sh, ring, ones);
        if constexpr (LOADING == BULK)
            if (warp == MULTIPLIER + 1) bulk_role<F>(a, sh, ring_bytes, lane);
        if constexpr (F::PAIRED)
            if (warp == MULTIPLIER + 1 && lane == 0) pair_role<F>(a, sh, ring_bytes, rank);
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

}  // namespace grouped

#endif
