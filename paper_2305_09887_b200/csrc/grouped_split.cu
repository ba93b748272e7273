// Grouped products (grouped_linear.cu) of fp32 rows on the tensor cores.
//
// A value is split into three bf16 numbers (8 + 8 + 8 bits, the whole significand) and a product is six MMAs; the three left out are
// below 2^-22 of it.  The tensor cores truncate when they accumulate: a stage of 32 terms starts a fresh accumulator, the five small
// products first, and is then added up in registers, rounded to nearest.
//
// The matrices are split beforehand, once a call, into planes in the scratch, and come by bulk-tensor loads in forward and dx; in dw
// both operands are rows.  The rows' values are split by the warps, which do everything in turn: split the next stage's values
// (which wait in registers) into shared memory, request the ones after, take their columns of the stage before from tensor memory
// and add them up.  When those are there, that stage's place in the ring and its accumulator are free again; warp 0 issues the MMAs,
// warp 1 the loads of W.  All these steps are short and wait for one another, so two blocks share an SM, each on tiles of 128 x 128
// (dw: 128 x 64): one block of twice the width on the SM, which splits less, took 127 us for 200,000 x 128 -> 256 and 220 for the
// 256 x 47 gradient of as many rows (two: 103).
//
// Bound by the chain of these steps, not by the six MMAs (47 us) or the bytes (48) of the first: 200,000 x 128 -> 256 125 us, its dx 133, the
// gradient of 256 x 256 295 (90 TFLOP/s of fp32 products).  Of the first, shared memory's data path is busy for 62 % of the cycles, the
// tensor pipes for 29 %, memory for 24 %, and instructions are issued in 35 %; of the 256 x 47 gradient 46, 15, 34 and 46 %.  The dx kernels
// spill 16 bytes a thread, the others nothing.
#include "grouped_linear.cuh"
#include "split.cuh"

RTMA_BOUNDS_TU()

namespace {

using namespace grouped;

constexpr int BM = 128, BK = 32, WARPS = 8, THREADS = 32 * WARPS, BLOCKS_PER_SM = SPLIT_BLOCKS_PER_SM;
constexpr int A_STAGES = 2, W_STAGES = 2;

template <int MODE>
struct Form {
    static constexpr bool W_BULK = MODE != WEIGHT_GRADIENT;           // the right operand is W and comes as planes
    static constexpr int BN = W_BULK ? 128 : SPLIT_DW_COLUMNS;
    static constexpr int COLUMNS = BN / 2, HALVES = COLUMNS / 32;      // of the accumulator that a warp drains, 32 at a time
    static constexpr int A_PLANE = BM * BK * 2, B_PLANE = BN * BK * 2;
    static constexpr int RING_BYTES = A_STAGES * 3 * A_PLANE + (W_BULK ? W_STAGES : A_STAGES) * 3 * B_PLANE;
    static constexpr int DYNAMIC_BYTES = RING_BYTES + 1024;
};

// fp32 matrices -> planes [part][3][d_in][ld] (ld: d_out rounded up to 8)
__global__ void __launch_bounds__(256) split_planes_kernel(const float* __restrict__ W, int64_t w_stride, int parts, int d_in, int d_out, int granule,
                                                           __nv_bfloat16* __restrict__ planes) {
    wait_for_kernel_before();
    const int units = (d_out + 7) / 8;
    const int64_t ld = 8 * (int64_t)units, matrix = ld * d_in, total = (int64_t)parts * d_in * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / units;
        const int u = (int)(i - row * units);
        const int64_t part = row / d_in, r = row - part * d_in;
        Eight<float> x;
        x.load(W + part * w_stride + r * d_out + 8 * u, min(8, d_out - 8 * u), granule);
        uint4 p[3];
        split_eight(reinterpret_cast<const uint32_t(&)[8]>(x.w), p);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(planes + (3 * part + k) * matrix + r * ld + 8 * u) = p[k];
    }
}

// One operand's values of a thread: PIECES units of eight, where they come from and where in a plane they go.
//   ALONG (K-major, 64-byte rows of 32 terms, 64-byte swizzle): unit t % 4 of rows t / 4 + (THREADS / 4) i
//   across (MN-major, atoms of 64 columns x 32 terms, 128-byte swizzle): unit t % U of terms t / U + (THREADS / U) i, U = columns / 8
template <bool ALONG, int COLUMNS>
struct Place {
    static constexpr int U = ALONG ? 4 : COLUMNS / 8, STEP = THREADS / U, PIECES = (ALONG ? BM : BK) / STEP;
    int row, unit;
    __device__ __forceinline__ explicit Place(int t) : row(t / U), unit(t % U) {}
    __device__ __forceinline__ uint32_t in_plane(int i) const {
        const int r = row + STEP * i;
        if constexpr (ALONG) return r * 64 + ((unit ^ ((r >> 1) & 3)) << 4);
        return (unit >> 3) * 4096 + r * 128 + (((unit & 7) ^ (r & 7)) << 4);
    }
};

// The walk of a thread down one operand's stages.
template <int MODE, bool IS_B>
struct Rows {
    static constexpr bool ALONG = MODE != WEIGHT_GRADIENT;
    typedef Place<ALONG, IS_B ? Form<MODE>::BN : BM> P;
    const float* p;  // this thread's first value of the tile
    int near, cols;  // along: rows from this thread's first on, terms;  across: terms from this thread's first on, columns
    __device__ __forceinline__ void open(const LinearArgs& a, const Walk<MODE, BM, BK>& w, const P& at) {
        const float* base = static_cast<const float*>(IS_B ? a.B : a.A);
        const int64_t ld = IS_B ? a.ldb : a.lda;
        p = base + (w.row0 + at.row) * ld + 8 * at.unit;
        if constexpr (ALONG) {
            near = w.rows - at.row;
            cols = w.k_end - 8 * at.unit;
        } else {
            const int c = IS_B ? w.n0 : w.m0;
            p += c;
            near = w.k_end - at.row;
            cols = (IS_B ? a.d_out : a.d_in) - c - 8 * at.unit;
        }
    }
    template <bool EASY>
    __device__ __forceinline__ void load(const LinearArgs& a, int k0, int i, Eight<float>& to) const {
        const float* from;
        int valid;
        if constexpr (ALONG) {
            from = p + P::STEP * i * (IS_B ? a.ldb : a.lda) + k0;
            valid = P::STEP * i < near ? cols - k0 : 0;
        } else {
            const int k = k0 + P::STEP * i;
            from = p + k * (IS_B ? a.ldb : a.lda);
            valid = k < near ? cols : 0;
        }
        if constexpr (EASY) {  // 16-byte boundaries, widths of whole 16 bytes
            uint32_t* q = reinterpret_cast<uint32_t*>(to.w);
            if (valid >= 8 && (IS_B ? a.vb : a.va) == 32) {
                asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]), "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7])
                             : "l"(from));
            } else {
                to.w[0] = to.w[1] = make_uint4(0u, 0u, 0u, 0u);
                if (valid > 0) to.w[0] = *reinterpret_cast<const uint4*>(from);
                if (valid > 4) to.w[1] = *reinterpret_cast<const uint4*>(from + 4);
            }
        } else {
            to.load(from, max(0, min(8, valid)), IS_B ? a.vb : a.va);
        }
    }
};

template <int MODE>
struct SplitShared : Shared {
    uint64_t w_full[W_STAGES];
    Walk<MODE, BM, BK> ahead;  // the stage of W that is fetched next, and its place: one thread's
    int ahead_slot;
    bool ahead_left;
};

// The stage's matrix by one thread, into its place in the ring.
template <int MODE>
__device__ __forceinline__ void load_w(const LinearArgs& a, SplitShared<MODE>& sh, uint8_t* to, int slot, const Walk<MODE, BM, BK>& w) {
    uint64_t* bar = &sh.w_full[slot];
    uint8_t* dst = to + slot * 3 * Form<MODE>::B_PLANE;
    const int z = a.w_stride ? 3 * w.part : 0;
    if constexpr (MODE == FORWARD) {  // atoms of 64 columns, their three planes behind one another
        const int atoms = (a.BN + 63) / 64;
        tc::mbar_arrive_expect_tx(bar, atoms * 3 * 4096);
        for (int i = 0; i < atoms; ++i) tc::tma_load_3d(dst + i * 3 * 4096, &a.map_b, bar, w.n0 + 64 * i, w.k0, z);
    } else {
        tc::mbar_arrive_expect_tx(bar, a.BN * 64 * 3);
        tc::tma_load_3d(dst, &a.map_b, bar, w.k0, w.n0, z);
    }
}

__device__ __forceinline__ uint64_t describe(uint32_t lbo, uint32_t sbo, bool narrow) {  // narrow: 64-byte swizzle
    return ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(sbo >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)(narrow ? 4 : 2) << 61);
}

template <int MODE>
__device__ __forceinline__ void multiply(const LinearArgs& a, uint32_t d, uint32_t sa, uint32_t sb, int terms) {
    typedef Form<MODE> F;
    constexpr bool A_ACROSS = MODE == WEIGHT_GRADIENT, B_ACROSS = MODE != INPUT_GRADIENT;
    const uint32_t idesc = tc::idesc_bf16(128, a.BN, A_ACROSS, B_ACROSS);
    const uint64_t da = (A_ACROSS ? describe(4096, 1024, false) : describe(16, 512, true)) + (sa >> 4);
    const uint64_t db = (MODE == INPUT_GRADIENT ? describe(16, 512, true) : describe(MODE == FORWARD ? 3 * 4096 : 4096, 1024, false)) + (sb >> 4);
    constexpr uint32_t a_step = A_ACROSS ? 128 : 2, b_step = B_ACROSS ? 128 : 2;  // 16 terms further
    constexpr uint32_t ap = F::A_PLANE >> 4;
    const uint32_t bp = MODE == FORWARD ? 4096 >> 4 : MODE == INPUT_GRADIENT ? (uint32_t)a.BN * 4 : F::B_PLANE >> 4;
    const bool two = terms > 16;
    tc::mma_by_warp(d, da + 2 * ap, db, idesc, 0u);
    tc::mma_by_warp(d, da, db + 2 * bp, idesc, 1u);
    tc::mma_by_warp(d, da + ap, db + bp, idesc, 1u);
    tc::mma_by_warp(d, da + ap, db, idesc, 1u);
    tc::mma_by_warp(d, da, db + bp, idesc, 1u);
    if (two) {
        const uint64_t x = da + a_step, y = db + b_step;
        tc::mma_by_warp(d, x + 2 * ap, y, idesc, 1u);
        tc::mma_by_warp(d, x, y + 2 * bp, idesc, 1u);
        tc::mma_by_warp(d, x + ap, y + bp, idesc, 1u);
        tc::mma_by_warp(d, x + ap, y, idesc, 1u);
        tc::mma_by_warp(d, x, y + bp, idesc, 1u);
        tc::mma_by_warp(d, x, y, idesc, 1u);
    }
    tc::mma_by_warp(d, da, db, idesc, 1u);
}

// 32 columns of a warp's rows (one per lane).  A lane writes its own row, as many bytes at a time as lie on a boundary: nothing is
// waited for, where bulk stores through the little shared memory there is left held the warps up (248 -> 129 us for 200,000 x 128 ->
// 256).
__device__ __forceinline__ void put_rows(float* out, int64_t ldo, int granule, const float (&v)[32], int rows, int cols, int lane) {
    if (lane >= rows) return;
    out += lane * ldo;
    if (granule == 32 && cols % 8 == 0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (8 * q < cols)
                asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + 8 * q), "f"(v[8 * q]), "f"(v[8 * q + 1]), "f"(v[8 * q + 2]),
                             "f"(v[8 * q + 3]), "f"(v[8 * q + 4]), "f"(v[8 * q + 5]), "f"(v[8 * q + 6]), "f"(v[8 * q + 7])
                             : "memory");
        }
    } else if (granule >= 16 && cols % 4 == 0) {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (4 * q < cols) *reinterpret_cast<float4*>(out + 4 * q) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < cols) out[j] = v[j];
    }
}

template <int MODE, int EASY>
__device__ __forceinline__ void work(const LinearArgs& a, SplitShared<MODE>& sh, uint8_t* ring_bytes) {
    typedef Form<MODE> F;
    typedef Walk<MODE, BM, BK> W;
    constexpr bool DW = MODE == WEIGHT_GRADIENT;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, quarter = warp & 3, group = warp >> 2;
    const uint32_t ring = tc::smem_u32(ring_bytes);
    constexpr int A_STAGE = 3 * F::A_PLANE, B_STAGE = 3 * F::B_PLANE;
    uint8_t* const b_bytes = ring_bytes + A_STAGES * A_STAGE;
    const uint32_t b_ring = ring + A_STAGES * A_STAGE;
    const typename Rows<MODE, false>::P place_a(t);
    const typename Rows<MODE, true>::P place_b(t);
    Rows<MODE, false> rows_a;
    Rows<MODE, true> rows_b;
    Eight<float> held_a[Rows<MODE, false>::P::PIECES], held_b[1];
    static_assert(!DW || Rows<MODE, true>::P::PIECES == 1, "one piece of dY a thread");
    // this warp's rows and columns of the accumulator
    const int out_m = 32 * quarter, out_c = F::COLUMNS * group;
    const uint32_t tmem = sh.tmem_base + ((uint32_t)out_m << 16) + out_c;
    const bool drains = out_c < a.BN;
    BiasHolder<float> bias{sh.bias + 64 * warp};
    float total[F::HALVES][32], sums[8];
    auto clear_total = [&]() {
#pragma unroll
        for (int h = 0; h < F::HALVES; ++h)
#pragma unroll
            for (int j = 0; j < 32; ++j) total[h][j] = 0.f;
    };
    clear_total();
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[j] = 0.f;

    // Stages are followed by their tile and first term; what else a tile has is looked up where it is needed (kept in registers for
    // the stage that is split, the one that is drained and the one that is fetched it does not fit).
    int tile = blockIdx.x, k0 = 0, k_end, out_tile = tile, out_k0 = 0, out_end, part = 0;  // part: not behind the drained tile's
    {
        W w;
        if (!w.first(a, sh)) return;
        k_end = out_end = w.k_end;
        rows_a.open(a, w, place_a);
        if constexpr (DW) rows_b.open(a, w, place_b);
    }
#pragma unroll
    for (int i = 0; i < Rows<MODE, false>::P::PIECES; ++i) rows_a.template load<(EASY & 1) != 0>(a, 0, i, held_a[i]);
    if constexpr (DW) rows_b.template load<(EASY & 2) != 0>(a, 0, 0, held_b[0]);
    if (F::W_BULK && t == 32) {
        bool some = sh.ahead.first(a, sh);
        for (int s = 0; s < W_STAGES && some; ++s) {
            load_w<MODE>(a, sh, b_bytes, s, sh.ahead);
            some = sh.ahead.next(a, sh);
        }
        sh.ahead_left = some;
        sh.ahead_slot = 0;
    }
    auto K = [&](int end) { return MODE == FORWARD ? a.d_in : MODE == INPUT_GRADIENT ? a.d_out : end; };
    uint32_t stage = 0;  // that is split next; one that has been split waits to be drained
    auto drain = [&]() {  // stage - 1: its accumulator, what follows from its place being free, and a finished tile's results
        const uint32_t before = stage - 1;
        if (!wait_for(&sh.acc_full[before & 1], before >> 1 & 1, sh, a.error_word)) return false;
        __syncwarp();
        tc::tc_fence_after_sync();
#pragma unroll
        for (int h = 0; h < F::HALVES; ++h) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[8];
                tc::tmem_load_32x8(tmem + (before & 1) * F::BN + 32 * h + 8 * q, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) total[h][8 * q + j] += v[j];
            }
        }
        tc::tc_fence_before_sync();
        if (F::W_BULK && t == 32 && sh.ahead_left) {
            load_w<MODE>(a, sh, b_bytes, sh.ahead_slot, sh.ahead);
            sh.ahead_slot = sh.ahead_slot + 1 == W_STAGES ? 0 : sh.ahead_slot + 1;
            sh.ahead_left = sh.ahead.next(a, sh);
        }
        out_k0 += BK;
        if (out_k0 < K(out_end)) return true;
        if (drains) {
            W out;
            out.tile = out_tile;
            out.part = part;
            out.at(a, sh);
            part = out.part;
            const int N = MODE == INPUT_GRADIENT ? a.d_in : MODE == FORWARD ? a.d_out : (int)a.ldo;  // (dw: the slots' rows are padded)
            const int rows = min(32, (DW ? min(BM, a.d_in - out.m0) : out.rows) - out_m);
            const int64_t row0 = (DW ? (int64_t)out.row_tile * (a.d_in + a.bias_rows) + out.m0 : out.row0) + out_m;
            if (MODE == FORWARD && a.bias) bias.fetch(a, out.part, out.n0, F::HALVES * group, 1, min(F::HALVES * (group + 1), (a.BN + 31) / 32), lane);
#pragma unroll
            for (int h = 0; h < F::HALVES; ++h) {
                const int c = out.n0 + out_c + 32 * h, cols = min(min(32, a.BN - out_c - 32 * h), N - c);
                if (rows > 0 && cols > 0) {
                    if (MODE == FORWARD && a.bias) bias.add(total[h], h);
                    put_rows(static_cast<float*>(a.out) + row0 * a.ldo + c, a.ldo, a.go, total[h], rows, cols, lane);
                }
            }
        }
        clear_total();
        out_k0 = 0;
        out_tile += gridDim.x;
        if constexpr (DW) {
            W out;
            out.tile = out_tile;
            out.part = part;
            if (out.at(a, sh)) out_end = out.k_end;
        }
        return true;
    };
    bool more = true;
    while (more) {
        const int terms = min(BK, K(k_end) - k0), this_tile = tile;
        const bool tile_ends = k0 + BK >= K(k_end);
        k0 += BK;
        if (tile_ends) {
            W w;
            w.tile = tile += gridDim.x;
            w.part = part;
            k0 = 0;
            more = w.at(a, sh);
            if (more) {
                if constexpr (DW) k_end = w.k_end;
                rows_a.open(a, w, place_a);
                if constexpr (DW) rows_b.open(a, w, place_b);
            }
        }
        const uint32_t slot = stage & 1, sa = ring + slot * A_STAGE;
#pragma unroll
        for (int i = 0; i < Rows<MODE, false>::P::PIECES; ++i) {
            uint4 planes[3];
            split_eight(reinterpret_cast<const uint32_t(&)[8]>(held_a[i].w), planes);
#pragma unroll
            for (int k = 0; k < 3; ++k) store_16(sa + k * F::A_PLANE + place_a.in_plane(i), planes[k]);
        }
        if constexpr (DW) {
            uint4 planes[3];
            float v[8];
            held_b[0].values(v);
            add_eight(sums, v);
            split_eight(reinterpret_cast<const uint32_t(&)[8]>(held_b[0].w), planes);
#pragma unroll
            for (int k = 0; k < 3; ++k) store_16(b_ring + slot * B_STAGE + k * F::B_PLANE + place_b.in_plane(0), planes[k]);
        }
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&sh.full[slot]);
        if (warp == 0) {
            const uint32_t round = stage / W_STAGES, w_slot = stage - round * W_STAGES;
            if (!wait_for(&sh.full[slot], stage >> 1 & 1, sh, a.error_word)) return;
            if (F::W_BULK && !wait_for(&sh.w_full[w_slot], round & 1, sh, a.error_word)) return;
            tc::tc_fence_after_sync();
            __syncwarp();
            multiply<MODE>(a, sh.tmem_base + slot * F::BN, sa, b_ring + (F::W_BULK ? w_slot : slot) * B_STAGE, terms);
            tc::commit_by_warp(&sh.acc_full[slot]);
        }
        if (more) {  // (before the fence they would be waited for there)
#pragma unroll
            for (int i = 0; i < Rows<MODE, false>::P::PIECES; ++i) rows_a.template load<(EASY & 1) != 0>(a, k0, i, held_a[i]);
            if constexpr (DW) rows_b.template load<(EASY & 2) != 0>(a, k0, 0, held_b[0]);
        }
        if constexpr (DW) {
            if (tile_ends) {  // four terms' threads of a warp hold the same columns
                W w;
                w.tile = this_tile;
                w.part = part;
                w.at(a, sh);
                float* to = static_cast<float*>(a.out) + ((int64_t)w.row_tile * (a.d_in + a.bias_rows) + a.d_in + warp) * a.ldo;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float s = sums[j] + __shfl_xor_sync(0xffffffffu, sums[j], 8);
                    s += __shfl_xor_sync(0xffffffffu, s, 16);
                    const int c = 8 * place_b.unit + j;
                    if (w.m0 == 0 && lane < 8 && c < a.BN && w.n0 + c < a.d_out) to[w.n0 + c] = s;
                    sums[j] = 0.f;
                }
            }
        }
        if (stage > 0 && !drain()) return;
        ++stage;
    }
    drain();
}

template <int MODE, int EASY>
__global__ void __launch_bounds__(THREADS, BLOCKS_PER_SM) split_kernel(const __grid_constant__ LinearArgs a) {
    typedef Form<MODE> F;
    static_assert(BLOCKS_PER_SM * (F::DYNAMIC_BYTES + sizeof(SplitShared<MODE>) + 1024) <= SMEM_MOST + 1024, "shared memory of a block");
    extern __shared__ uint8_t raw[];
    __shared__ SplitShared<MODE> sh;
    uint8_t* ring = raw + ((1024u - (tc::smem_u32(raw) & 1023u)) & 1023u);
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int s = 0; s < 2; ++s) {
            tc::mbar_init(&sh.full[s], WARPS);
            tc::mbar_init(&sh.acc_full[s], 1);
        }
        for (int s = 0; s < W_STAGES; ++s) tc::mbar_init(&sh.w_full[s], 1);
        sh.abort = 0;
        tc::fence_barrier_init();
        if (F::W_BULK) tc::prefetch_tensormap(&a.map_b);
    }
    if (warp == 0) {
        tc::tmem_alloc(&sh.tmem_base, 2 * F::BN);
        tc::tmem_relinquish();
    }
    wait_for_kernel_before();
    lay_out<MODE, THREADS, BK>(a, sh);
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    work<MODE, EASY>(a, sh, ring);
    __syncwarp();
    if (*reinterpret_cast<volatile int*>(&sh.abort)) __nanosleep(1000000);  // a wait ran out: copies and MMAs under way land before the block ends
    tc::tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc(sh.tmem_base, 2 * F::BN);
    }
}

template <int MODE, int EASY>
int32_t launch_form(rtma_ctx* ctx, const LinearArgs& a, unsigned grid, bool& configured, cudaStream_t stream) {
    if (!configured) {
        RTMA_CUDA(ctx, cudaFuncSetAttribute(split_kernel<MODE, EASY>, cudaFuncAttributeMaxDynamicSharedMemorySize, Form<MODE>::DYNAMIC_BYTES));
        configured = true;
    }
    launch_kernel(split_kernel<MODE, EASY>, grid, THREADS, Form<MODE>::DYNAMIC_BYTES, stream, a);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

template <int MODE>
int32_t launch_mode(rtma_ctx* ctx, LinearArgs& a, void* planes, int cls, cudaStream_t stream) {
    if (MODE != WEIGHT_GRADIENT) {
        const int parts = a.w_stride ? a.G : 1, units = (a.d_out + 7) / 8;
        const int64_t ld = 8 * (int64_t)units, work = (int64_t)parts * a.d_in * units, blocks = ceil_div(work, 256);
        if (!make_tensor_map_16bit(&a.map_b, true, planes, 3 * (uint64_t)parts, a.d_in, a.d_out, ld, ld * a.d_in, MODE == FORWARD ? BK : a.BN,
                                   MODE == FORWARD ? 64 : 32, 3))
            return rtma_fail(ctx, RTMA_ERR_CUDA, "grouped product: no tensor map for %d matrices of %d x %d", parts, a.d_in, a.d_out);
        KernelScope ks(ctx, KC_WEIGHT_PREP, stream);
        launch_kernel(split_planes_kernel, (unsigned)(blocks < 16 * ctx->sm_count ? blocks : 16 * ctx->sm_count), 256, 0, stream,
                      static_cast<const float*>(a.B), a.w_stride, parts, a.d_in, a.d_out, a.vb, static_cast<__nv_bfloat16*>(planes));
        RTMA_LAUNCH_CHECK(ctx);
    }
    const int64_t tiles = a.tiles * a.m_tiles * a.n_tiles;
    const int64_t places = (int64_t)BLOCKS_PER_SM * ctx->sm_count;
    const unsigned grid = (unsigned)(tiles < places ? tiles : places);
    // operands on 16-byte boundaries with widths of whole 16 bytes are loaded without a case for every value
    const bool easy_a = a.va >= 16 && (MODE == INPUT_GRADIENT ? a.d_out : a.d_in) % 4 == 0, easy_b = a.vb >= 16 && a.d_out % 4 == 0;
    bool* configured = ctx->split_configured + 4 * MODE;
    KernelScope ks(ctx, cls, stream);
    if constexpr (MODE == WEIGHT_GRADIENT) {
        if (easy_b) return easy_a ? launch_form<MODE, 3>(ctx, a, grid, configured[3], stream) : launch_form<MODE, 2>(ctx, a, grid, configured[2], stream);
    }
    return easy_a ? launch_form<MODE, 1>(ctx, a, grid, configured[1], stream) : launch_form<MODE, 0>(ctx, a, grid, configured[0], stream);
}

}  // namespace

size_t split_planes_bytes(const LinearArgs& a) {
    return (size_t)3 * 2 * (a.w_stride ? a.G : 1) * a.d_in * ((a.d_out + 7) / 8 * 8);
}

int32_t launch_split(rtma_ctx* ctx, int mode, LinearArgs& a, void* planes, int cls, cudaStream_t stream) {
    const int64_t tiles = a.tiles * a.m_tiles * a.n_tiles;
    if (tiles >= (int64_t(1) << 30)) return rtma_fail(ctx, RTMA_ERR_OVERFLOW, "grouped product: %lld tiles", (long long)tiles);
    return mode == FORWARD ? launch_mode<FORWARD>(ctx, a, planes, cls, stream)
           : mode == INPUT_GRADIENT ? launch_mode<INPUT_GRADIENT>(ctx, a, planes, cls, stream)
                                    : launch_mode<WEIGHT_GRADIENT>(ctx, a, planes, cls, stream);
}
