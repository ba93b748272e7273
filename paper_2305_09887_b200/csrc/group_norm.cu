// Group norm over channels that lie last, with the activation and dropout behind it, and its gradient.
//   xhat = (x - mean) * rstd, u = gamma xhat + beta, h = act(u), y = dropout(h)
// mean and rstd = 1 / sqrt(var + eps) are those of a set of C / groups neighbouring channels, of one row (scope 0) or of all rows
// of a part (scope 1); gamma, beta and the PReLU slope are the part's own (or shared).  Backward, with m values in a set:
//   dh = dropout(dy), du = dh act'(u), dgamma = sum du xhat, dbeta = sum du, dslope = sum_{u <= 0} dh u,
//   dx = rstd (gamma du - (S1 + xhat S2) / m),  S1 = sum gamma du, S2 = sum gamma du xhat over the set.
// A thread keeps eight neighbouring channels and walks down the rows of a tile (a run of rows of one part); what is summed over
// rows is left per tile and added up in a fixed order by a second kernel, so results do not depend on which block ran when.
#include <algorithm>
#include <type_traits>

#include "activation.cuh"
#include "rows.cuh"

RTMA_BOUNDS_TU()

namespace {

constexpr int NORM_THREADS = 256;
constexpr int NORM_MAX_CHANNELS = 8 * NORM_THREADS;

struct NormArgs {
    const int64_t* offsets;
    int64_t n;
    int G, C, groups, per_set, units, rows_at_once, pitch;  // per_set = C / groups; units of eight channels; rows a block works on at a time;
                                                           // lanes of a row where warps keep rows to themselves (0: they do not)
    bool straddles;  // sets share units, two at most
    bool wide;       // a set's lanes are in several warps, or may be
    int within;      // sets of 1, 2 or 4 channels, which share units but do not straddle them; otherwise 0
    int tile_rows;
    int64_t tiles;   // at most so many
    int act;
    float eps;
    const void *X, *dY;
    void* Y;  // forward: y; backward: dx
    int64_t ldx, lddy, ldy;
    int vx, vdy, vy;  // granules of the rows (bytes)
    const float *gamma, *beta, *slope;
    int64_t gamma_stride, beta_stride, slope_stride;
    DropArgs drop;
    float* stats;    // [row or part][groups][2]
    float2* pieces;  // part scope, forward: [tile][groups] (mean, sum of squared differences)
    float* partial;  // backward: [tile][2 C + 1]: sums of du, of du xhat, of the slope's gradient
    float* sums;     // backward: [part][2 C + 1]
    float *dgamma, *dbeta, *dslope;
    int64_t dgamma_stride, dbeta_stride, dslope_stride;
};

// (x - mean) * rstd of a pair.  The difference first, so that a mean much larger than the deviation costs no digits: with the mean
// folded into x rstd + (-mean rstd) a set of equal values, whose rstd is 1 / sqrt(eps), is off by half a step of mean rstd.  The
// subtraction costs the row gradient of 16-bit rows 2 % (1M x 256 in one set 314 -> 320 us).
struct Standard {
    f2 r, m;
    __device__ __forceinline__ void set(float mean0, float rstd0, float mean1, float rstd1) {
        r = pack2(rstd0, rstd1);
        m = pack2(-mean0, -mean1);
    }
    __device__ __forceinline__ f2 operator()(f2 x) const { return mul2(add2(x, m), r); }
};

__device__ __forceinline__ uint32_t id_of(const NormArgs& a, int64_t r) {
    return a.drop.ids ? (uint32_t)__ldg(a.drop.ids + r) : (uint32_t)r;
}

// A thread's place in a block and its channels' parameters.
struct Lane {
    int u, y, valid;  // unit, row within those worked on at a time, channels that exist
    bool active;
    __device__ __forceinline__ explicit Lane(const NormArgs& a) {
        y = threadIdx.x / a.units;
        u = threadIdx.x - y * a.units;
        active = y < a.rows_at_once;
        valid = active ? min(8, a.C - 8 * u) : 0;
    }
};
__device__ __forceinline__ void load_params(const float* p, int64_t stride, int part, int u, int valid, float missing, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = p && j < valid ? __ldg(p + part * stride + 8 * u + j) : (j < valid ? missing : 0.f);
}
__device__ __forceinline__ void load_params(const float* p, int64_t stride, int part, int u, int valid, float missing, f2 (&v)[4]) {
    float x[8];
    load_params(p, stride, part, u, valid, missing, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2(x[2 * i], x[2 * i + 1]);
}

// The lanes that share one set's sum: a power of two, so many that a block's threads cover `sets` sets.
__device__ __forceinline__ int lanes_per_set(int per_set, int sets) {
    int l = 32;
    while (l > 1 && (l > per_set || l * sets > NORM_THREADS)) l >>= 1;
    return l;
}
__device__ __forceinline__ float lane_sum(float x, int lanes) {
    for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// ---- statistics of a row ---------------------------------------------------------------------------
// Any sets, of any size, through shared memory; called for those of 3, 5, 6 or 7 channels.  Far from memory's pace, for the block waits for
// all its rows twice: 500,000 x 60 in 20 sets, bf16, 188 us, gradient 300.
__device__ __forceinline__ int row_pitch(const NormArgs& a) { return a.units * 8; }

template <class T>
__global__ void __launch_bounds__(NORM_THREADS) norm_rows_kernel(const NormArgs a) {
    extern __shared__ float shared[];
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int pitch = row_pitch(a);
    float* vals = shared;                                                        // [rows_at_once][pitch]
    float2* stat = reinterpret_cast<float2*>(vals + a.rows_at_once * pitch);     // [rows_at_once][groups]
    const Lane at(a);
    const int pairs = a.rows_at_once * a.groups, L = lanes_per_set(a.per_set, pairs), sets_at_once = NORM_THREADS / L;
    const T* X = static_cast<const T*>(a.X);
    T* Y = static_cast<T*>(a.Y);
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const int part = part_of_tile(tile_start, a.G, tile);
        int64_t begin, end;
        part_rows(a.offsets, a.n, part, begin, end);
        begin += (int64_t)(tile - tile_start[part]) * a.tile_rows;
        end = min(end, begin + a.tile_rows);
        float gam[8], bet[8];
        load_params(a.gamma, a.gamma_stride, part, at.u, at.valid, 1.f, gam);
        load_params(a.beta, a.beta_stride, part, at.u, at.valid, 0.f, bet);
        const float slope = a.slope ? __ldg(a.slope + part * a.slope_stride) : 0.f;
        for (int64_t r0 = begin; r0 < end; r0 += a.rows_at_once) {
            const int64_t r = r0 + at.y;
            const bool here = at.active && r < end;
            float v[8];
            if (here) {
                Eight<T> x;
                x.load(X + r * a.ldx + 8 * at.u, at.valid, a.vx);
                x.values(v);
                float4* to = reinterpret_cast<float4*>(vals + at.y * pitch + 8 * at.u);
                to[0] = make_float4(v[0], v[1], v[2], v[3]);
                to[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
            __syncthreads();
            for (int s0 = 0; s0 < pairs; s0 += sets_at_once) {  // pair = row, set
                const int pair = s0 + threadIdx.x / L, l = threadIdx.x % L;
                const int y = pair / a.groups, set = pair - y * a.groups;
                const bool ok = pair < pairs && r0 + y < end;
                const float* p = vals + y * pitch + set * a.per_set;
                float s = 0.f;
                if (ok) for (int i = l; i < a.per_set; i += L) s += p[i];
                const float mean = lane_sum(s, L) / (float)a.per_set;
                s = 0.f;
                if (ok) for (int i = l; i < a.per_set; i += L) s += (p[i] - mean) * (p[i] - mean);
                s = lane_sum(s, L);
                if (ok && l == 0) {
                    const float2 st = make_float2(mean, 1.f / sqrtf(s / (float)a.per_set + a.eps));
                    stat[pair] = st;
                    if (a.stats) *reinterpret_cast<float2*>(a.stats + 2 * ((r0 + y) * a.groups + set)) = st;
                }
            }
            __syncthreads();
            if (here) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j < at.valid) {
                        const float2 st = stat[at.y * a.groups + (8 * at.u + j) / a.per_set];
                        v[j] = fmaf((v[j] - st.x) * st.y, gam[j], bet[j]);
                    }
                }
                f2 w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1]);
                activate(a.act, slope, w);
                if (a.drop.threshold) drop_pairs(a.drop, id_of(a, r), at.u, w);
                store_pairs(Y + r * a.ldy + 8 * at.u, w, at.valid, a.vy);
            }
        }
    }
}

// dh (in du) -> du and x (in xhat) -> xhat of eight channels; returns the slope's gradient
__device__ __forceinline__ float back(const NormArgs& a, int64_t r, int u, const Standard (&st)[4], const f2 (&gam)[4], const f2 (&bet)[4],
                                      float slope, f2 (&xhat)[4], f2 (&du)[4]) {
    if (a.drop.threshold) drop_pairs(a.drop, id_of(a, r), u, du);
    f2 pre[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        xhat[i] = st[i](xhat[i]);
        pre[i] = fma2(xhat[i], gam[i], bet[i]);
    }
    return activate_back(a.act, slope, pre, du);
}

// Sums over a block's rows of (du, du xhat) of a thread's eight channels from c0 on, written to the tile's slot.  Threads pitch apart
// hold the same channels, rows_at_once of them.
__device__ __forceinline__ void leave_sums(const NormArgs& a, int tile, int c0, int y, int pitch, int rows_at_once, const f2 (&sb)[4], const f2 (&sg)[4], float* red) {
    int top = 1;
    while (top < rows_at_once) top <<= 1;
    float* out = a.partial + (int64_t)tile * (2 * a.C + 1);
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(kind == 0 ? sb[i] : sg[i], red[2 * i * NORM_THREADS + threadIdx.x], red[(2 * i + 1) * NORM_THREADS + threadIdx.x]);
        for (int h = top >> 1; h > 0; h >>= 1) {
            __syncthreads();
            if (y < h && y + h < rows_at_once) {
#pragma unroll
                for (int j = 0; j < 8; ++j) red[j * NORM_THREADS + threadIdx.x] += red[j * NORM_THREADS + threadIdx.x + h * pitch];
            }
        }
        __syncthreads();
        if (y == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j < a.C) out[kind * a.C + c0 + j] = red[j * NORM_THREADS + threadIdx.x];
        }
    }
    __syncthreads();
}
__device__ __forceinline__ void leave_slope(const NormArgs& a, int tile, float ds, float* red) {
    red[threadIdx.x] = ds;
    for (int h = NORM_THREADS / 2; h > 0; h >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < h) red[threadIdx.x] += red[threadIdx.x + h];
    }
    __syncthreads();
    if (threadIdx.x == 0) a.partial[(int64_t)tile * (2 * a.C + 1) + 2 * a.C] = red[0];
    __syncthreads();
}

// 1 / sqrt(x) for x >= eps > 0: the approximation and a Newton step, within a unit in the last place (x y first: half of a number
// below 2^-126 loses bits).  0 for an infinite x, a variance that does not fit fp32.
__device__ __forceinline__ float inverse_root(float x) {
    const float y = rsqrtf(x);
    return x < __int_as_float(0x7f800000) ? y * fmaf(x * y, -0.5f * y, 1.5f) : y;
}

// A run of rows of one part.
struct Run {
    int part;
    int64_t begin, end;
    __device__ __forceinline__ Run(const NormArgs& a, const int32_t* tile_start, int tile) {
        part = part_of_tile(tile_start, a.G, tile);
        part_rows(a.offsets, a.n, part, begin, end);
        begin += (int64_t)(tile - tile_start[part]) * a.tile_rows;
        end = min(end, begin + a.tile_rows);
    }
};

// ---- rows whose sets are runs of lanes -------------------------------------------------------------
// A row lies in `pitch` lanes (a power of two, 256 at most), eight channels each; a set is the whole row or a power of two of
// neighbouring lanes, so its sums are exchanged within a warp, and only those of sets of more than 256 channels (WIDE) go through
// shared memory.  RB rows side by side hide one another's loads and shuffles.  Reads each row once; bound by instructions (two sums
// exchanged per row, the activation) at 4.7 to 6 TB/s: 2M x 128 in bf16 with ReLU 185 us, 200,000 x 1024 in 8 sets fp32 with SiLU 280;
// gradients of 200,000 x 256 in 8 sets, fp32 with dropout, 132 us and of 1M x 256 in bf16 320 (two rows of three kinds fill the 128 registers:
// of fp32 rows 56 bytes a thread are spilled, 64 with WIDE, 104 and 152 where units are not whole; 16-bit rows spill nothing).  With up to 16
// channels a lane instead (and shared memory above 512) these two and 500,000 x 512 took 132, 405 and 466 us.
// Sums over `lanes` lanes, in every lane.  WIDE: red, 8 floats per sum, is used by every other call.
template <bool WIDE, int N>
__device__ __forceinline__ void set_sums(float (&x)[N], int lanes, float* red) {
    for (int o = (WIDE ? 32 : lanes) >> 1; o > 0; o >>= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], o);
    }
    if constexpr (WIDE) {
        const int warp = threadIdx.x >> 5, first = warp & ~(lanes / 32 - 1);
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) red[8 * i + warp] = x[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = 0.f;
            for (int w = first; w < first + lanes / 32; ++w) x[i] += red[8 * i + w];
        }
    }
}

template <class T, bool FULL, bool WIDE>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_warp_rows_kernel(const NormArgs a) {
    constexpr int RB = 4;  // rows in flight
    __shared__ float red[2][8 * RB];
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int pitch = a.pitch, u = threadIdx.x & (pitch - 1), y = threadIdx.x / pitch, rows_at_once = NORM_THREADS / pitch;
    const bool whole = a.groups == 1;
    const int lanes = whole ? pitch : a.per_set / 8, lanes_log = 31 - __clz(lanes);  // of a set
    const float inv = 1.f / (float)a.per_set;
    const int valid = max(0, min(8, a.C - 8 * u));
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const Run run(a, tile_start, tile);
        f2 gam[4], bet[4];
        load_params(a.gamma, a.gamma_stride, run.part, u, valid, 1.f, gam);
        load_params(a.beta, a.beta_stride, run.part, u, valid, 0.f, bet);
        const float slope = a.slope ? __ldg(a.slope + run.part * a.slope_stride) : 0.f;
        Eight<T> raw[RB];  // the next rows are on their way while these are worked on
        int left = (int)(run.end - run.begin), asked = left - y;  // rows from this step's first on; from this lane's next request on
        const T* x = static_cast<const T*>(a.X) + (run.begin + y) * a.ldx + 8 * u;
        T* out = static_cast<T*>(a.Y) + (run.begin + y) * a.ldy + 8 * u;
        int64_t r = run.begin + y;
        const int64_t x_step = rows_at_once * a.ldx, out_step = rows_at_once * a.ldy;
        auto request = [&]() {
#pragma unroll
            for (int b = 0; b < RB; ++b, x += x_step) load_unit<FULL>(raw[b], x, b * rows_at_once < asked, valid, a.vx);
            asked -= RB * rows_at_once;
        };
        request();
        for (; left > 0; left -= RB * rows_at_once) {  // the same number of times in every lane
            f2 v[RB][4];
            float mean[RB], rstd[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b) pairs_of(raw[b], v[b]);
            request();
#pragma unroll
            for (int b = 0; b < RB; ++b) mean[b] = halves_sum(add2(add2(v[b][0], v[b][1]), add2(v[b][2], v[b][3])));  // what is not there reads as zero
            set_sums<WIDE>(mean, lanes, red[0]);
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                mean[b] *= inv;
                const f2 minus = pack2(-mean[b], -mean[b]);
                f2 q = 0ull;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[b][i] = add2(v[b][i], minus);
                    f2 t = v[b][i];
                    if (!FULL && valid < 8) {  // channels that are not there do not count
                        float t0, t1;
                        unpack2(t, t0, t1);
                        t = pack2(2 * i < valid ? t0 : 0.f, 2 * i + 1 < valid ? t1 : 0.f);
                    }
                    q = fma2(t, t, q);
                }
                rstd[b] = halves_sum(q);
            }
            set_sums<WIDE>(rstd, lanes, red[1]);
#pragma unroll
            for (int b = 0; b < RB; ++b) rstd[b] = inverse_root(fmaf(rstd[b], inv, a.eps));
#pragma unroll
            for (int b = 0; b < RB; ++b, out += out_step, r += rows_at_once) {
                if (y + b * rows_at_once >= left || (!FULL && valid == 0)) continue;
                if (a.stats && (u & (lanes - 1)) == 0)
                    *reinterpret_cast<float2*>(a.stats + 2 * (r * a.groups + (u >> lanes_log))) = make_float2(mean[b], rstd[b]);
                const f2 r2 = pack2(rstd[b], rstd[b]);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[b][i] = fma2(mul2(v[b][i], r2), gam[i], bet[i]);
                activate(a.act, slope, v[b]);
                if (a.drop.threshold) drop_pairs(a.drop, id_of(a, r), u, v[b]);
                store_unit<FULL>(out, v[b], valid, a.vy);
            }
        }
    }
}

template <class T, bool FULL, bool WIDE>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_warp_rows_grad_kernel(const NormArgs a) {
    constexpr int RB = 2;  // rows in flight
    __shared__ float shared[8 * NORM_THREADS];
    __shared__ float red[2][16 * RB];
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int pitch = a.pitch, u = threadIdx.x & (pitch - 1), y = threadIdx.x / pitch, rows_at_once = NORM_THREADS / pitch;
    const bool whole = a.groups == 1;
    const int lanes = whole ? pitch : a.per_set / 8, lanes_log = 31 - __clz(lanes);
    const float inv = 1.f / (float)a.per_set;
    const int valid = max(0, min(8, a.C - 8 * u));
    int turn = 0;
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const Run run(a, tile_start, tile);
        f2 gam[4], bet[4], sb[4], sg[4];
        float ds = 0.f;
        load_params(a.gamma, a.gamma_stride, run.part, u, valid, 1.f, gam);
        load_params(a.beta, a.beta_stride, run.part, u, valid, 0.f, bet);
#pragma unroll
        for (int i = 0; i < 4; ++i) sb[i] = sg[i] = 0ull;
        const float slope = a.slope ? __ldg(a.slope + run.part * a.slope_stride) : 0.f;
        Eight<T> rx[RB], rd[RB];
        float2 rs[RB];
        int left = (int)(run.end - run.begin), asked = left - y;
        const T* x = static_cast<const T*>(a.X) + (run.begin + y) * a.ldx + 8 * u;
        const T* dy = static_cast<const T*>(a.dY) + (run.begin + y) * a.lddy + 8 * u;
        const float* stat = a.stats + 2 * ((run.begin + y) * a.groups + (u >> lanes_log));
        T* out = static_cast<T*>(a.Y) + (run.begin + y) * a.ldy + 8 * u;
        int64_t r = run.begin + y;
        const int64_t x_step = rows_at_once * a.ldx, dy_step = rows_at_once * a.lddy, out_step = rows_at_once * a.ldy;
        const int stat_step = 2 * rows_at_once * a.groups;
        auto request = [&]() {
#pragma unroll
            for (int b = 0; b < RB; ++b, x += x_step, dy += dy_step, stat += stat_step) {
                const bool here = b * rows_at_once < asked;
                load_unit<FULL>(rx[b], x, here, valid, a.vx);
                load_unit<FULL>(rd[b], dy, here, valid, a.vdy);
                rs[b] = here && (FULL || valid) ? *reinterpret_cast<const float2*>(stat) : make_float2(0.f, 0.f);
            }
            asked -= RB * rows_at_once;
        };
        request();
        for (; left > 0; left -= RB * rows_at_once) {
            f2 xh[RB][4], du[RB][4];
            float s12[2 * RB], rstd[RB];  // sums over the set of gamma du, and of gamma du xhat
            Standard st[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                pairs_of(rx[b], xh[b]);
                pairs_of(rd[b], du[b]);
                st[b].set(rs[b].x, rs[b].y, rs[b].x, rs[b].y);
                rstd[b] = rs[b].y;
            }
            request();
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                if (a.drop.threshold) drop_pairs(a.drop, y + b * rows_at_once < left ? id_of(a, r + b * rows_at_once) : 0u, u, du[b]);
                f2 pre[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    xh[b][i] = st[b](xh[b][i]);
                    pre[i] = fma2(xh[b][i], gam[i], bet[i]);
                }
                ds += activate_back(a.act, slope, pre, du[b]);
                f2 t1 = 0ull, t2 = 0ull;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sb[i] = add2(sb[i], du[b][i]);
                    sg[i] = fma2(du[b][i], xh[b][i], sg[i]);
                    du[b][i] = mul2(du[b][i], gam[i]);
                    t1 = add2(t1, du[b][i]);
                    t2 = fma2(du[b][i], xh[b][i], t2);
                }
                s12[2 * b] = halves_sum(t1);
                s12[2 * b + 1] = halves_sum(t2);
            }
            set_sums<WIDE>(s12, lanes, red[turn]);
            turn ^= 1;
#pragma unroll
            for (int b = 0; b < RB; ++b, out += out_step, r += rows_at_once) {
                if (y + b * rows_at_once >= left || (!FULL && valid == 0)) continue;
                const float n1 = -inv * s12[2 * b], n2 = -inv * s12[2 * b + 1];
                const f2 m1 = pack2(n1, n1), m2 = pack2(n2, n2), r2 = pack2(rstd[b], rstd[b]);
#pragma unroll
                for (int i = 0; i < 4; ++i) du[b][i] = mul2(r2, fma2(xh[b][i], m2, add2(du[b][i], m1)));
                store_unit<FULL>(out, du[b], valid, a.vy);
            }
        }
        leave_sums(a, tile, 8 * u, y, pitch, rows_at_once, sb, sg, shared);
        leave_slope(a, tile, ds, shared);
    }
}

// ---- rows whose sets share units ---------------------------------------------
// Sets of eight channels or more that do not end with a unit: a unit's channels belong to one set or to two.  A row lies in `pitch`
// lanes as above; a set's sum grows from lane to lane in a scan that starts anew where a set begins, is complete in the lane with the
// set's last channel and fetched from there.  WIDE: rows of more than 256 channels; the warps' scans are joined in shared memory.
// Bound by instructions: 1M x 100 in 4 sets, fp16, 230 us, gradient 287 (through shared memory,
// by the kernels for all other sets, 550 and 990); 1M x 240 in 10 sets, fp32, 369 and 582.  WIDE by its barriers, too: 500,000 x 300 in
// 3 sets, fp16, 745 and 888 (853 and 1408), x 384 in 8 sets, fp32, 703 and 787.
struct Straddle {
    int set, first;   // set of the unit's first channel, how many of its channels are in it
    bool begins, two; // the set begins with the unit; another one begins within it
    int start;        // the lane where the unit's first set begins
    int back;         // lanes from where the unit's last set begins
    int end0, end1;   // lanes where the two sums are complete
    __device__ __forceinline__ Straddle(const NormArgs& a, int u) {
        const int c = 8 * u;
        const bool there = c < a.C;
        set = there ? c / a.per_set : 0;
        const int c0 = set * a.per_set;
        first = there ? min(8, c0 + a.per_set - c) : 8;
        begins = !there || c == c0;
        start = there ? c0 >> 3 : u;
        two = first < 8 && c + first < a.C;
        back = begins || first < 8 ? 0 : u - (c0 >> 3);
        end0 = there ? (c0 + a.per_set - 1) >> 3 : u;
        end1 = two ? (c0 + 2 * a.per_set - 1) >> 3 : end0;
    }
    __device__ __forceinline__ f2 choose(int i, float in_first, float in_second) const {  // for channels 2 i and 2 i + 1
        return pack2(2 * i < first ? in_first : in_second, 2 * i + 1 < first ? in_first : in_second);
    }
    // a unit's sums over the channels of its two sets
    __device__ __forceinline__ void part(const f2 (&v)[4], float& lo, float& hi) const {
        lo = hi = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x, y;
            unpack2(v[i], x, y);
            lo += (2 * i < first ? x : 0.f) + (2 * i + 1 < first ? y : 0.f);
            hi += (2 * i < first ? 0.f : x) + (2 * i + 1 < first ? 0.f : y);
        }
    }
    // ... become the sets' sums.  WIDE: ends is 8 floats per sum, sums NORM_THREADS; everything before is read when a call is through.
    template <bool WIDE, int N>
    __device__ __forceinline__ void join(float (&lo)[N], float (&hi)[N], int u, int pitch, int far, float* ends, float* sums) const {
        const int width = WIDE ? 32 : pitch, lane = u & 31, within = WIDE ? min(back, lane) : back;
        float open[N];  // of the set that goes on behind the unit
#pragma unroll
        for (int i = 0; i < N; ++i) open[i] = first < 8 ? hi[i] : lo[i];
        for (int o = 1; o <= far && o < 32; o <<= 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float x = __shfl_up_sync(0xffffffffu, open[i], o, width);
                if (o <= within) open[i] += x;
            }
        }
        const int warp = threadIdx.x >> 5, mine = u >> 5, row = warp - mine;  // of the block, of the row; the row's first
        if constexpr (WIDE) {
            if (lane == 31) {
#pragma unroll
                for (int i = 0; i < N; ++i) ends[8 * i + warp] = open[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i)
                for (int w = (u - back) >> 5; w < mine; ++w) open[i] += ends[8 * i + row + w];
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float before = __shfl_up_sync(0xffffffffu, open[i], 1, width);
            if (WIDE && lane == 0) {
                before = 0.f;
                for (int w = start >> 5; w < mine; ++w) before += ends[8 * i + row + w];
            }
            const float all = begins ? lo[i] : before + lo[i];
            if constexpr (WIDE) {
                sums[NORM_THREADS * i + threadIdx.x] = all;
            } else {
                lo[i] = __shfl_sync(0xffffffffu, all, end0, pitch);
                hi[i] = __shfl_sync(0xffffffffu, all, end1, pitch);
            }
        }
        if constexpr (WIDE) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                lo[i] = sums[NORM_THREADS * i + threadIdx.x - u + end0];
                hi[i] = sums[NORM_THREADS * i + threadIdx.x - u + end1];
            }
        }
    }
};

template <class T, bool FULL, bool WIDE>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_straddle_rows_kernel(const NormArgs a) {
    constexpr int RB = 2;  // rows in flight
    __shared__ float ends[WIDE ? 8 * RB : 1], sums[WIDE ? NORM_THREADS * RB : 1];
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int pitch = a.pitch, u = threadIdx.x & (pitch - 1), y = threadIdx.x / pitch, rows_at_once = NORM_THREADS / pitch;
    const int valid = max(0, min(8, a.C - 8 * u)), far = (a.per_set + 7) / 8;
    const Straddle sets(a, u);
    const float inv = 1.f / (float)a.per_set;
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const Run run(a, tile_start, tile);
        f2 gam[4], bet[4];
        load_params(a.gamma, a.gamma_stride, run.part, u, valid, 1.f, gam);
        load_params(a.beta, a.beta_stride, run.part, u, valid, 0.f, bet);
        const float slope = a.slope ? __ldg(a.slope + run.part * a.slope_stride) : 0.f;
        Eight<T> raw[RB];
        int left = (int)(run.end - run.begin), asked = left - y;
        const T* x = static_cast<const T*>(a.X) + (run.begin + y) * a.ldx + 8 * u;
        T* out = static_cast<T*>(a.Y) + (run.begin + y) * a.ldy + 8 * u;
        int64_t r = run.begin + y;
        const int64_t x_step = rows_at_once * a.ldx, out_step = rows_at_once * a.ldy;
        auto request = [&]() {
#pragma unroll
            for (int b = 0; b < RB; ++b, x += x_step) load_unit<FULL>(raw[b], x, b * rows_at_once < asked && valid, valid, a.vx);
            asked -= RB * rows_at_once;
        };
        request();
        for (; left > 0; left -= RB * rows_at_once) {  // the same number of times in every lane
            f2 v[RB][4];
            float mean0[RB], mean1[RB], rstd0[RB], rstd1[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                pairs_of(raw[b], v[b]);
                sets.part(v[b], mean0[b], mean1[b]);  // (what is not there reads as zero)
            }
            request();
            sets.join<WIDE>(mean0, mean1, u, pitch, far, ends, sums);
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                mean0[b] *= inv;
                mean1[b] *= inv;
                f2 q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[b][i] = add2(v[b][i], sets.choose(i, -mean0[b], -mean1[b]));
                    float q0, q1;
                    unpack2(mul2(v[b][i], v[b][i]), q0, q1);
                    q[i] = pack2(2 * i < valid ? q0 : 0.f, 2 * i + 1 < valid ? q1 : 0.f);
                }
                sets.part(q, rstd0[b], rstd1[b]);
            }
            sets.join<WIDE>(rstd0, rstd1, u, pitch, far, ends, sums);
#pragma unroll
            for (int b = 0; b < RB; ++b, out += out_step, r += rows_at_once) {
                rstd0[b] = inverse_root(fmaf(rstd0[b], inv, a.eps));
                rstd1[b] = inverse_root(fmaf(rstd1[b], inv, a.eps));
                if (y + b * rows_at_once >= left || valid == 0) continue;
                if (a.stats) {
                    float2* st = reinterpret_cast<float2*>(a.stats) + r * a.groups + sets.set;
                    if (sets.begins) st[0] = make_float2(mean0[b], rstd0[b]);
                    if (sets.two) st[1] = make_float2(mean1[b], rstd1[b]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) v[b][i] = fma2(mul2(v[b][i], sets.choose(i, rstd0[b], rstd1[b])), gam[i], bet[i]);
                activate(a.act, slope, v[b]);
                if (a.drop.threshold) drop_pairs(a.drop, id_of(a, r), u, v[b]);
                store_unit<FULL>(out, v[b], valid, a.vy);
            }
        }
    }
}

template <class T, bool FULL, bool WIDE>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_straddle_rows_grad_kernel(const NormArgs a) {
    constexpr int RB = 1;  // rows in flight: two do not fit the registers (1M x 100 in 4 sets, fp16: 320 us instead of 287)
    __shared__ float ends[WIDE ? 16 * RB : 1], sums[WIDE ? 2 * NORM_THREADS * RB : 1];
    __shared__ float shared[8 * NORM_THREADS];
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int pitch = a.pitch, u = threadIdx.x & (pitch - 1), y = threadIdx.x / pitch, rows_at_once = NORM_THREADS / pitch;
    const int valid = max(0, min(8, a.C - 8 * u)), far = (a.per_set + 7) / 8;
    const Straddle sets(a, u);
    const float inv = 1.f / (float)a.per_set;
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const Run run(a, tile_start, tile);
        f2 gam[4], bet[4], sb[4], sg[4];
        float ds = 0.f;
        load_params(a.gamma, a.gamma_stride, run.part, u, valid, 1.f, gam);
        load_params(a.beta, a.beta_stride, run.part, u, valid, 0.f, bet);
#pragma unroll
        for (int i = 0; i < 4; ++i) sb[i] = sg[i] = 0ull;
        const float slope = a.slope ? __ldg(a.slope + run.part * a.slope_stride) : 0.f;
        Eight<T> rx[RB], rd[RB];
        float2 s0[RB], s1[RB];
        int left = (int)(run.end - run.begin), asked = left - y;
        const T* x = static_cast<const T*>(a.X) + (run.begin + y) * a.ldx + 8 * u;
        const T* dy = static_cast<const T*>(a.dY) + (run.begin + y) * a.lddy + 8 * u;
        const float2* stat = reinterpret_cast<const float2*>(a.stats) + (run.begin + y) * a.groups + sets.set;
        T* out = static_cast<T*>(a.Y) + (run.begin + y) * a.ldy + 8 * u;
        int64_t r = run.begin + y;
        const int64_t x_step = rows_at_once * a.ldx, dy_step = rows_at_once * a.lddy, out_step = rows_at_once * a.ldy;
        auto request = [&]() {
#pragma unroll
            for (int b = 0; b < RB; ++b, x += x_step, dy += dy_step, stat += rows_at_once * a.groups) {
                const bool here = b * rows_at_once < asked && valid;
                load_unit<FULL>(rx[b], x, here, valid, a.vx);
                load_unit<FULL>(rd[b], dy, here, valid, a.vdy);
                s0[b] = here ? stat[0] : make_float2(0.f, 0.f);
                s1[b] = here && sets.two ? stat[1] : make_float2(0.f, 0.f);
            }
            asked -= RB * rows_at_once;
        };
        request();
        for (; left > 0; left -= RB * rows_at_once) {
            f2 xh[RB][4], du[RB][4];
            float lo[2 * RB], hi[2 * RB], rstd0[RB], rstd1[RB];  // sums over the sets of gamma du, and of gamma du xhat
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                pairs_of(rx[b], xh[b]);
                pairs_of(rd[b], du[b]);
                const uint32_t id = a.drop.threshold && y + b * rows_at_once < left ? id_of(a, r + b * rows_at_once) : 0u;
                if (a.drop.threshold) drop_pairs(a.drop, id, u, du[b]);
                f2 pre[4], t[4];
                rstd0[b] = s0[b].y;
                rstd1[b] = s1[b].y;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f2 r2 = sets.choose(i, rstd0[b], rstd1[b]);
                    xh[b][i] = mul2(add2(xh[b][i], sets.choose(i, -s0[b].x, -s1[b].x)), r2);
                    pre[i] = fma2(xh[b][i], gam[i], bet[i]);
                }
                ds += activate_back(a.act, slope, pre, du[b]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sb[i] = add2(sb[i], du[b][i]);
                    sg[i] = fma2(du[b][i], xh[b][i], sg[i]);
                    du[b][i] = mul2(du[b][i], gam[i]);
                    t[i] = mul2(du[b][i], xh[b][i]);
                }
                sets.part(du[b], lo[2 * b], hi[2 * b]);
                sets.part(t, lo[2 * b + 1], hi[2 * b + 1]);
            }
            request();
            sets.join<WIDE>(lo, hi, u, pitch, far, ends, sums);
#pragma unroll
            for (int b = 0; b < RB; ++b, out += out_step, r += rows_at_once) {
                if (y + b * rows_at_once >= left || valid == 0) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f2 m1 = sets.choose(i, -inv * lo[2 * b], -inv * hi[2 * b]), m2 = sets.choose(i, -inv * lo[2 * b + 1], -inv * hi[2 * b + 1]);
                    du[b][i] = mul2(sets.choose(i, rstd0[b], rstd1[b]), fma2(xh[b][i], m2, add2(du[b][i], m1)));
                }
                store_unit<FULL>(out, du[b], valid, a.vy);
            }
        }
        leave_sums(a, tile, 8 * u, y, pitch, rows_at_once, sb, sg, shared);
        leave_slope(a, tile, ds, shared);
    }
}

// ---- rows whose sets lie within units --------------------------------------------------------------
// Sets of P = 1, 2 or 4 channels: a lane has all of a set, nothing is exchanged.  (Channels that are not there are whole sets.)
// 1M x 64 in 32 sets, bf16, 117 to 127 us, gradient 130 (through shared memory 435 and 645); 200,000 x 128 in 32 sets, fp32, 47 and 73.
// (Of the gradient's forms only that of single fp32 channels in rows that are not whole units spills: 32 bytes a thread.)
template <int P>
__device__ __forceinline__ void sums_within(f2 (&x)[4]) {  // every channel's set's sum
#pragma unroll
    for (int i = 0; i < 4; i += P == 4 ? 2 : 1) {
        if constexpr (P >= 2) {
            const float s = halves_sum(P == 4 ? add2(x[i], x[i + (P == 4)]) : x[i]);
            x[i] = x[i + (P == 4)] = pack2(s, s);
        }
    }
}

template <class T, int P, bool FULL>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_unit_rows_kernel(const NormArgs a) {
    constexpr int RB = 2;  // rows in flight
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int pitch = a.pitch, u = threadIdx.x & (pitch - 1), y = threadIdx.x / pitch, rows_at_once = NORM_THREADS / pitch;
    const int valid = max(0, min(8, a.C - 8 * u));
    const f2 inv = pack2(1.f / P, 1.f / P), minus = pack2(-1.f, -1.f);
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const Run run(a, tile_start, tile);
        f2 gam[4], bet[4];
        load_params(a.gamma, a.gamma_stride, run.part, u, valid, 1.f, gam);
        load_params(a.beta, a.beta_stride, run.part, u, valid, 0.f, bet);
        const float slope = a.slope ? __ldg(a.slope + run.part * a.slope_stride) : 0.f;
        Eight<T> raw[RB];
        int left = (int)(run.end - run.begin) - y, asked = left;
        const T* x = static_cast<const T*>(a.X) + (run.begin + y) * a.ldx + 8 * u;
        T* out = static_cast<T*>(a.Y) + (run.begin + y) * a.ldy + 8 * u;
        int64_t r = run.begin + y;
        const int64_t x_step = rows_at_once * a.ldx, out_step = rows_at_once * a.ldy;
        auto request = [&]() {
#pragma unroll
            for (int b = 0; b < RB; ++b, x += x_step) load_unit<FULL>(raw[b], x, b * rows_at_once < asked && valid, valid, a.vx);
            asked -= RB * rows_at_once;
        };
        request();
        for (; left > 0; left -= RB * rows_at_once) {
            f2 v[RB][4];
#pragma unroll
            for (int b = 0; b < RB; ++b) pairs_of(raw[b], v[b]);
            request();
#pragma unroll
            for (int b = 0; b < RB; ++b, out += out_step, r += rows_at_once) {
                if (b * rows_at_once >= left || valid == 0) continue;
                f2 mean[4], q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) mean[i] = v[b][i];
                sums_within<P>(mean);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mean[i] = mul2(mean[i], inv);
                    v[b][i] = fma2(mean[i], minus, v[b][i]);
                    q[i] = mul2(v[b][i], v[b][i]);
                }
                sums_within<P>(q);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float q0, q1;
                    unpack2(q[i], q0, q1);
                    q[i] = pack2(inverse_root(fmaf(q0, 1.f / P, a.eps)), inverse_root(fmaf(q1, 1.f / P, a.eps)));
                }
                if (a.stats) {
                    float2* st = reinterpret_cast<float2*>(a.stats) + r * a.groups + 8 / P * u;
#pragma unroll
                    for (int j = 0; j < 8; j += P) {
                        float m0, m1, s0, s1;
                        unpack2(mean[j / 2], m0, m1);
                        unpack2(q[j / 2], s0, s1);
                        if (j < valid) st[j / P] = make_float2(j & 1 ? m1 : m0, j & 1 ? s1 : s0);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) v[b][i] = fma2(mul2(v[b][i], q[i]), gam[i], bet[i]);
                activate(a.act, slope, v[b]);
                if (a.drop.threshold) drop_pairs(a.drop, id_of(a, r), u, v[b]);
                store_unit<FULL>(out, v[b], valid, a.vy);
            }
        }
    }
}

template <class T, int P, bool FULL>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_unit_rows_grad_kernel(const NormArgs a) {
    __shared__ float shared[8 * NORM_THREADS];
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int pitch = a.pitch, u = threadIdx.x & (pitch - 1), y = threadIdx.x / pitch, rows_at_once = NORM_THREADS / pitch;
    const int valid = max(0, min(8, a.C - 8 * u));
    const f2 minus_inv = pack2(-1.f / P, -1.f / P);
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const Run run(a, tile_start, tile);
        f2 gam[4], bet[4], sb[4], sg[4];
        float ds = 0.f;
        load_params(a.gamma, a.gamma_stride, run.part, u, valid, 1.f, gam);
        load_params(a.beta, a.beta_stride, run.part, u, valid, 0.f, bet);
#pragma unroll
        for (int i = 0; i < 4; ++i) sb[i] = sg[i] = 0ull;
        const float slope = a.slope ? __ldg(a.slope + run.part * a.slope_stride) : 0.f;
        Eight<T> rx, rd;
        float2 rs[8 / P];
        int left = (int)(run.end - run.begin) - y, asked = left;
        const T* x = static_cast<const T*>(a.X) + (run.begin + y) * a.ldx + 8 * u;
        const T* dy = static_cast<const T*>(a.dY) + (run.begin + y) * a.lddy + 8 * u;
        const float2* stat = reinterpret_cast<const float2*>(a.stats) + (run.begin + y) * a.groups + 8 / P * u;
        T* out = static_cast<T*>(a.Y) + (run.begin + y) * a.ldy + 8 * u;
        int64_t r = run.begin + y;
        const int64_t x_step = rows_at_once * a.ldx, dy_step = rows_at_once * a.lddy, out_step = rows_at_once * a.ldy;
        auto request = [&]() {
            const bool here = asked > 0 && valid;
            load_unit<FULL>(rx, x, here, valid, a.vx);
            load_unit<FULL>(rd, dy, here, valid, a.vdy);
#pragma unroll
            for (int j = 0; j < 8 / P; ++j) rs[j] = here && j * P < valid ? stat[j] : make_float2(0.f, 0.f);
            x += x_step;
            dy += dy_step;
            stat += rows_at_once * a.groups;
            asked -= rows_at_once;
        };
        request();
        for (; left > 0; left -= rows_at_once, out += out_step, r += rows_at_once) {
            f2 xh[4], du[4], rstd[4], pre[4], t1[4], t2[4];
            pairs_of(rx, xh);
            pairs_of(rd, du);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 s0 = rs[2 * i / P], s1 = rs[(2 * i + 1) / P];
                Standard st;
                st.set(s0.x, s0.y, s1.x, s1.y);
                rstd[i] = pack2(s0.y, s1.y);
                xh[i] = st(xh[i]);
                pre[i] = fma2(xh[i], gam[i], bet[i]);
            }
            request();
            if (a.drop.threshold) drop_pairs(a.drop, id_of(a, r), u, du);
            ds += activate_back(a.act, slope, pre, du);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sb[i] = add2(sb[i], du[i]);
                sg[i] = fma2(du[i], xh[i], sg[i]);
                t1[i] = du[i] = mul2(du[i], gam[i]);
                t2[i] = mul2(du[i], xh[i]);
            }
            sums_within<P>(t1);
            sums_within<P>(t2);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                du[i] = mul2(rstd[i], fma2(xh[i], mul2(t2[i], minus_inv), fma2(t1[i], minus_inv, du[i])));
            if (valid) store_unit<FULL>(out, du, valid, a.vy);
        }
        leave_sums(a, tile, 8 * u, y, pitch, rows_at_once, sb, sg, shared);
        leave_slope(a, tile, ds, shared);
    }
}

template <class T>
__global__ void __launch_bounds__(NORM_THREADS) norm_rows_grad_kernel(const NormArgs a) {
    extern __shared__ float shared[];
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int pitch = row_pitch(a);
    float2* vals = reinterpret_cast<float2*>(shared);                    // [rows_at_once][pitch] (gamma du, gamma du xhat)
    float2* stat = vals + (NORM_THREADS * 8);                            // [rows_at_once][groups]
    const Lane at(a);
    const int pairs = a.rows_at_once * a.groups, L = lanes_per_set(a.per_set, pairs), sets_at_once = NORM_THREADS / L;
    T* Y = static_cast<T*>(a.Y);
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const int part = part_of_tile(tile_start, a.G, tile);
        int64_t begin, end;
        part_rows(a.offsets, a.n, part, begin, end);
        begin += (int64_t)(tile - tile_start[part]) * a.tile_rows;
        end = min(end, begin + a.tile_rows);
        f2 gam[4], bet[4], sb[4], sg[4];
        float ds = 0.f;
        load_params(a.gamma, a.gamma_stride, part, at.u, at.valid, 1.f, gam);
        load_params(a.beta, a.beta_stride, part, at.u, at.valid, 0.f, bet);
        const float slope = a.slope ? __ldg(a.slope + part * a.slope_stride) : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sb[i] = sg[i] = 0ull;
        for (int64_t r0 = begin; r0 < end; r0 += a.rows_at_once) {
            const int64_t r = r0 + at.y;
            const bool here = at.active && r < end;
            f2 xhat[4], du[4];
            float rstd[8];
            if (here) {
                float mean[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 st = j < at.valid ? *reinterpret_cast<const float2*>(a.stats + 2 * (r * a.groups + (8 * at.u + j) / a.per_set)) : make_float2(0.f, 0.f);
                    mean[j] = st.x;
                    rstd[j] = st.y;
                }
                Standard st[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) st[i].set(mean[2 * i], rstd[2 * i], mean[2 * i + 1], rstd[2 * i + 1]);
                Eight<T> x, d;
                x.load(static_cast<const T*>(a.X) + r * a.ldx + 8 * at.u, at.valid, a.vx);
                d.load(static_cast<const T*>(a.dY) + r * a.lddy + 8 * at.u, at.valid, a.vdy);
                pairs_of(x, xhat);
                pairs_of(d, du);
                ds += back(a, r, at.u, st, gam, bet, slope, xhat, du);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sb[i] = add2(sb[i], du[i]);
                    sg[i] = fma2(du[i], xhat[i], sg[i]);
                    du[i] = mul2(du[i], gam[i]);
                    float t0, t1, q0, q1;
                    unpack2(du[i], t0, t1);
                    unpack2(mul2(du[i], xhat[i]), q0, q1);
                    *reinterpret_cast<float4*>(&vals[at.y * pitch + 8 * at.u + 2 * i]) = make_float4(t0, q0, t1, q1);
                }
            }
            __syncthreads();
            for (int s0 = 0; s0 < pairs; s0 += sets_at_once) {
                const int pair = s0 + threadIdx.x / L, l = threadIdx.x % L;
                const int y = pair / a.groups, set = pair - y * a.groups;
                const bool ok = pair < pairs && r0 + y < end;
                const float2* p = vals + y * pitch + set * a.per_set;
                float s1 = 0.f, s2 = 0.f;
                if (ok) {
                    for (int i = l; i < a.per_set; i += L) {
                        s1 += p[i].x;
                        s2 += p[i].y;
                    }
                }
                s1 = lane_sum(s1, L);
                s2 = lane_sum(s2, L);
                if (ok && l == 0) stat[pair] = make_float2(s1 / (float)a.per_set, s2 / (float)a.per_set);
            }
            __syncthreads();
            if (here) {
                float t[8], x[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    unpack2(du[i], t[2 * i], t[2 * i + 1]);
                    unpack2(xhat[i], x[2 * i], x[2 * i + 1]);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j < at.valid) {
                        const float2 st = stat[at.y * a.groups + (8 * at.u + j) / a.per_set];
                        t[j] = rstd[j] * (t[j] - st.x - x[j] * st.y);
                    }
                }
                store_eight(Y + r * a.ldy + 8 * at.u, t, at.valid, a.vy);
            }
        }
        leave_sums(a, tile, 8 * at.u, at.active ? at.y : NORM_THREADS, a.units, a.rows_at_once, sb, sg, shared);
        leave_slope(a, tile, ds, shared);
    }
}

// ---- statistics of a part --------------------------------------------------------------------------
// (mean, sum of squared differences) of two disjoint samples joined (Chan, Golub and LeVeque)
__device__ __forceinline__ void join_moments(float& mean, float& m2, float n, float mean_b, float m2_b, float n_b) {
    const float d = mean_b - mean, share = n_b / (n + n_b);
    mean += d * share;
    m2 += m2_b + d * d * n * share;
}

// Mean and sum of squared differences of every set within a tile.  A thread joins four rows at a time to its channels' moments: the
// batch's mean costs no division, and a mean far from zero costs no digits.  2M x 128 in bf16: 110 us, 4.7 TB/s (instructions).
template <class T, bool FULL>
__global__ void __launch_bounds__(NORM_THREADS, FULL ? 3 : 2) norm_stats_kernel(const NormArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    __shared__ float s_mean[8 * NORM_THREADS], s_m2[8 * NORM_THREADS], s_count[NORM_THREADS];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const Lane at(a);
    const T* X = static_cast<const T*>(a.X);
    const int L = lanes_per_set(a.per_set, a.groups), sets_at_once = NORM_THREADS / L;
    constexpr int BATCH = 4;  // rows in flight
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const int part = part_of_tile(tile_start, a.G, tile);
        int64_t begin, end;
        part_rows(a.offsets, a.n, part, begin, end);
        begin += (int64_t)(tile - tile_start[part]) * a.tile_rows;
        end = min(end, begin + a.tile_rows);
        f2 mean[4], m2[4];
        float count = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) mean[i] = m2[i] = 0ull;
        if (at.active) {
            int64_t r = begin + at.y;
            const int64_t step = BATCH * (int64_t)a.rows_at_once;
            const f2 minus = pack2(-1.f, -1.f), part_of_batch = pack2(1.f / BATCH, 1.f / BATCH);
            Eight<T> x[BATCH];
            int asked = (int)(end - r);
            const T* from = X + r * a.ldx + 8 * at.u;
            const int64_t x_step = a.rows_at_once * a.ldx;
            auto request = [&]() {  // rows behind the last are not there
#pragma unroll
                for (int b = 0; b < BATCH; ++b, from += x_step) load_unit<FULL>(x[b], from, b * a.rows_at_once < asked, at.valid, a.vx);
                asked -= BATCH * a.rows_at_once;
            };
            request();
            for (; r + step - a.rows_at_once < end; r += step) {
                // moments of the batch about its own mean, then joined to the thread's
                const float share = BATCH / (count + BATCH), weight = count * share;
                const f2 share2 = pack2(share, share), weight2 = pack2(weight, weight);
                f2 v[BATCH][4];
#pragma unroll
                for (int b = 0; b < BATCH; ++b) pairs_of(x[b], v[b]);
                request();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f2 s = v[0][i];
#pragma unroll
                    for (int b = 1; b < BATCH; ++b) s = add2(s, v[b][i]);
                    s = mul2(s, part_of_batch);
                    f2 q = m2[i];
#pragma unroll
                    for (int b = 0; b < BATCH; ++b) {
                        const f2 d = fma2(s, minus, v[b][i]);
                        q = fma2(d, d, q);
                    }
                    const f2 d = fma2(mean[i], minus, s);
                    mean[i] = fma2(d, share2, mean[i]);
                    m2[i] = fma2(mul2(d, weight2), d, q);  // (in this order: a weight of 0 makes any finite d 0)
                }
                count += BATCH;
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (r + b * a.rows_at_once >= end) break;
                f2 v[4];
                pairs_of(x[b], v);
                const float share = 1.f / (count + 1.f), weight = count * share;
                const f2 share2 = pack2(share, share), weight2 = pack2(weight, weight);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f2 d = fma2(mean[i], minus, v[i]);
                    mean[i] = fma2(d, share2, mean[i]);
                    m2[i] = fma2(mul2(d, weight2), d, m2[i]);
                }
                count += 1.f;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unpack2(mean[i], s_mean[2 * i * NORM_THREADS + threadIdx.x], s_mean[(2 * i + 1) * NORM_THREADS + threadIdx.x]);
            unpack2(m2[i], s_m2[2 * i * NORM_THREADS + threadIdx.x], s_m2[(2 * i + 1) * NORM_THREADS + threadIdx.x]);
        }
        s_count[threadIdx.x] = count;
        int top = 1;
        while (top < a.rows_at_once) top <<= 1;
        for (int h = top >> 1; h > 0; h >>= 1) {
            __syncthreads();
            const int other = threadIdx.x + h * a.units;
            float n = 0.f, nb = 0.f;
            if (at.active && at.y < h && at.y + h < a.rows_at_once) {
                n = s_count[threadIdx.x];
                nb = s_count[other];
                if (nb > 0.f) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        join_moments(s_mean[j * NORM_THREADS + threadIdx.x], s_m2[j * NORM_THREADS + threadIdx.x], n,
                                     s_mean[j * NORM_THREADS + other], s_m2[j * NORM_THREADS + other], nb);
                }
                s_count[threadIdx.x] = n + nb;
            }
        }
        __syncthreads();
        const float rows = (float)(end - begin);
        for (int s0 = 0; s0 < a.groups; s0 += sets_at_once) {
            const int set = s0 + threadIdx.x / L, l = threadIdx.x % L;
            const bool ok = set < a.groups;
            const int c0 = set * a.per_set;
            const float first = ok ? s_mean[(c0 & 7) * NORM_THREADS + (c0 >> 3)] : 0.f;
            float s = 0.f;
            if (ok) for (int c = c0 + l; c < c0 + a.per_set; c += L) s += s_mean[(c & 7) * NORM_THREADS + (c >> 3)] - first;
            const float m = first + lane_sum(s, L) / (float)a.per_set;
            float q = 0.f;
            if (ok) {
                for (int c = c0 + l; c < c0 + a.per_set; c += L) {
                    const float d = s_mean[(c & 7) * NORM_THREADS + (c >> 3)] - m;
                    q += s_m2[(c & 7) * NORM_THREADS + (c >> 3)] + rows * d * d;
                }
            }
            q = lane_sum(q, L);
            if (ok && l == 0) a.pieces[(int64_t)tile * a.groups + set] = make_float2(m, q);
        }
        __syncthreads();
    }
}

// The tiles' moments of every (part, set) joined: a warp each, in a fixed order (8 us for 16 parts of 32 sets, most of it latency).
__global__ void __launch_bounds__(NORM_THREADS) norm_join_kernel(const NormArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int lane = threadIdx.x & 31;
    const int job = (int)(((int64_t)blockIdx.x * NORM_THREADS + threadIdx.x) >> 5);
    if (job >= a.G * a.groups) return;
    const int part = job / a.groups, set = job - part * a.groups;
    int64_t begin, end;
    part_rows(a.offsets, a.n, part, begin, end);
    const int t0 = tile_start[part], t1 = tile_start[part + 1];
    float2 st = make_float2(0.f, 1.f / sqrtf(a.eps));
    if (t1 > t0) {
        const float total = (float)(end - begin);
        const float2* p = a.pieces + set;
        const float first = p[(int64_t)t0 * a.groups].x;
        float s = 0.f;
        for (int t = t0 + lane; t < t1; t += 32) {
            const float rows = (float)min((int64_t)a.tile_rows, end - begin - (int64_t)(t - t0) * a.tile_rows);
            s += rows * (p[(int64_t)t * a.groups].x - first);
        }
        const float mean = first + lane_sum(s, 32) / total;
        float q = 0.f;
        for (int t = t0 + lane; t < t1; t += 32) {
            const float rows = (float)min((int64_t)a.tile_rows, end - begin - (int64_t)(t - t0) * a.tile_rows);
            const float2 v = p[(int64_t)t * a.groups];
            const float d = v.x - mean;
            q += v.y + rows * (float)a.per_set * d * d;
        }
        q = lane_sum(q, 32);
        st = make_float2(mean, 1.f / sqrtf(q / (total * (float)a.per_set) + a.eps));
    }
    if (lane == 0) *reinterpret_cast<float2*>(a.stats + 2 * ((int64_t)part * a.groups + set)) = st;
}

__device__ __forceinline__ void load_part_stats(const NormArgs& a, int part, const Lane& at, float (&mean)[8], float (&rstd)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 st = j < at.valid ? *reinterpret_cast<const float2*>(a.stats + 2 * ((int64_t)part * a.groups + (8 * at.u + j) / a.per_set)) : make_float2(0.f, 0.f);
        mean[j] = st.x;
        rstd[j] = st.y;
    }
}

// The second pass of part scope; 2M x 128 in bf16 with SiLU: 160 us (4 bytes a thread are spilled).  (Rows backwards, so that it starts with what the first pass read
// last, and loads and stores past the cache changed nothing: it is not memory alone that bounds it.)

// minus the mean, rstd gamma and beta of a thread's channels
__device__ __forceinline__ void load_coefficients(const NormArgs& a, int part, const Lane& at, f2 (&minus_mean)[4], f2 (&scale)[4], f2 (&bet)[4], float (&rstd)[8]) {
    float gam[8], mean[8];
    load_params(a.gamma, a.gamma_stride, part, at.u, at.valid, 1.f, gam);
    load_params(a.beta, a.beta_stride, part, at.u, at.valid, 0.f, bet);
    load_part_stats(a, part, at, mean, rstd);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        minus_mean[i] = pack2(-mean[2 * i], -mean[2 * i + 1]);
        scale[i] = pack2(rstd[2 * i] * gam[2 * i], rstd[2 * i + 1] * gam[2 * i + 1]);
    }
}
// x (in t) -> x - mean, dh (in du) -> du; returns the slope's gradient
__device__ __forceinline__ float back_centred(const NormArgs& a, int64_t r, int u, const f2 (&minus_mean)[4], const f2 (&scale)[4], const f2 (&bet)[4],
                                              float slope, f2 (&t)[4], f2 (&du)[4]) {
    if (a.drop.threshold) drop_pairs(a.drop, id_of(a, r), u, du);
    f2 pre[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t[i] = add2(t[i], minus_mean[i]);
        pre[i] = fma2(t[i], scale[i], bet[i]);
    }
    return activate_back(a.act, slope, pre, du);
}

template <class T, bool FULL>
__global__ void __launch_bounds__(NORM_THREADS, FULL ? 3 : 2) norm_apply_kernel(const NormArgs a) {
    constexpr int RB = 8 / sizeof(T);  // rows in flight
    constexpr float FOLD = 64.f;
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const Lane at(a);
    if (!at.active) return;
    const T* X = static_cast<const T*>(a.X);
    T* Y = static_cast<T*>(a.Y);
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const int part = part_of_tile(tile_start, a.G, tile);
        int64_t begin, end;
        part_rows(a.offsets, a.n, part, begin, end);
        begin += (int64_t)(tile - tile_start[part]) * a.tile_rows;
        end = min(end, begin + a.tile_rows);
        // u = (x - mean) scale + beta (see Standard), or x scale + (beta - mean scale) for 16-bit rows whose means are within FOLD deviations of zero:
        // the rounding of the sum in brackets, 2^-24 FOLD of a deviation, is then far below that of the result.  2M x 128 in bf16 with
        // SiLU 275 us, with the subtraction always 281; 500,000 x 256 in fp16 with dropout 181 and 190.
        f2 minus_mean[4], scale[4], bet[4];
        bool folds = sizeof(T) == 2;
        {
            float rstd[8];
            load_coefficients(a, part, at, minus_mean, scale, bet, rstd);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float m0, m1;
                unpack2(minus_mean[i], m0, m1);
                folds &= fabsf(m0) * rstd[2 * i] <= FOLD && fabsf(m1) * rstd[2 * i + 1] <= FOLD;
            }
            if (folds) {
#pragma unroll
                for (int i = 0; i < 4; ++i) bet[i] = fma2(minus_mean[i], scale[i], bet[i]);
            }
        }
        const float slope = a.slope ? __ldg(a.slope + part * a.slope_stride) : 0.f;
        Eight<T> x[RB];
        int64_t row = begin + at.y;
        int left = (int)(end - row), asked = left;
        const T* from = X + row * a.ldx + 8 * at.u;
        T* out = Y + row * a.ldy + 8 * at.u;
        const int64_t x_step = a.rows_at_once * a.ldx, out_step = a.rows_at_once * a.ldy;
        auto request = [&](int b) {
            load_unit<FULL>(x[b], from, asked > 0, at.valid, a.vx);
            from += x_step;
            asked -= a.rows_at_once;
        };
#pragma unroll
        for (int b = 0; b < RB; ++b) request(b);
        const auto rows = [&](auto folded) {
            while (left > 0) {
#pragma unroll
                for (int b = 0; b < RB; ++b, row += a.rows_at_once, out += out_step) {
                    if (left <= 0) break;
                    left -= a.rows_at_once;
                    f2 v[4];
                    pairs_of(x[b], v);
                    request(b);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = fma2(decltype(folded)::value ? v[i] : add2(v[i], minus_mean[i]), scale[i], bet[i]);
                    activate(a.act, slope, v);
                    if (a.drop.threshold) drop_pairs(a.drop, id_of(a, row), at.u, v);
                    store_unit<FULL>(out, v, at.valid, a.vy);
                }
            }
        };
        if (folds) rows(std::true_type{});
        else rows(std::false_type{});
    }
}

// The gradient of part scope in two passes, as the sums over a part have to be complete before any of its rows: 500,000 x 256 in
// bf16 with SiLU 262 us, 8 of them for joining the sums; the rows' pass works out du again (storing it would cost as many bytes).  Bound by
// the loads on their way: with two rows of 16-bit values in flight instead of four 281 us, without an activation 254 (four: 226).  The first
// kernel spills 32 bytes a thread of 16-bit rows and 16 of fp32 ones (up to 52 where units are not whole), the second 12 and 8 (up to 36).
template <class T, bool FULL>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_grad_sums_kernel(const NormArgs a) {
    constexpr int RB = 8 / sizeof(T);  // rows in flight
    __shared__ float shared[8 * NORM_THREADS];
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const Lane at(a);
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const int part = part_of_tile(tile_start, a.G, tile);
        int64_t begin, end;
        part_rows(a.offsets, a.n, part, begin, end);
        begin += (int64_t)(tile - tile_start[part]) * a.tile_rows;
        end = min(end, begin + a.tile_rows);
        // u = (x - mean) scale + beta; the sum of du xhat is rstd times that of du (x - mean)
        f2 minus_mean[4], scale[4], bet[4], sb[4], sg[4];
        float rstd[8], ds = 0.f;
        load_coefficients(a, part, at, minus_mean, scale, bet, rstd);
        const float slope = a.slope ? __ldg(a.slope + part * a.slope_stride) : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sb[i] = sg[i] = 0ull;
        if (at.active) {
            Eight<T> x[RB], d[RB];
            int64_t row = begin + at.y;
            int left = (int)(end - row), asked = left;
            const T* from = static_cast<const T*>(a.X) + row * a.ldx + 8 * at.u;
            const T* d_from = static_cast<const T*>(a.dY) + row * a.lddy + 8 * at.u;
            const int64_t x_step = a.rows_at_once * a.ldx, d_step = a.rows_at_once * a.lddy;
            auto request = [&](int b) {
                load_unit<FULL>(x[b], from, asked > 0, at.valid, a.vx);
                load_unit<FULL>(d[b], d_from, asked > 0, at.valid, a.vdy);
                from += x_step;
                d_from += d_step;
                asked -= a.rows_at_once;
            };
#pragma unroll
            for (int b = 0; b < RB; ++b) request(b);
            while (left > 0) {
#pragma unroll
                for (int b = 0; b < RB; ++b, row += a.rows_at_once) {
                    if (left <= 0) break;
                    left -= a.rows_at_once;
                    f2 t[4], du[4];
                    pairs_of(x[b], t);
                    pairs_of(d[b], du);
                    request(b);
                    ds += back_centred(a, row, at.u, minus_mean, scale, bet, slope, t, du);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        sb[i] = add2(sb[i], du[i]);
                        sg[i] = fma2(du[i], t[i], sg[i]);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float s0, s1;
            unpack2(sg[i], s0, s1);
            sg[i] = pack2(rstd[2 * i] == 0.f ? 0.f : s0 * rstd[2 * i], rstd[2 * i + 1] == 0.f ? 0.f : s1 * rstd[2 * i + 1]);  // (sums may be infinite)
        }
        leave_sums(a, tile, 8 * at.u, at.active ? at.y : NORM_THREADS, a.units, a.rows_at_once, sb, sg, shared);
        leave_slope(a, tile, ds, shared);
    }
}

template <class T, bool FULL>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_grad_apply_kernel(const NormArgs a) {
    constexpr int RB = 8 / sizeof(T);  // rows in flight
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    __shared__ float2 of_set[NORM_MAX_CHANNELS];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const Lane at(a);
    T* Y = static_cast<T*>(a.Y);
    const int L = lanes_per_set(a.per_set, a.groups), sets_at_once = NORM_THREADS / L;
    for (int tile = blockIdx.x; tile < tile_start[a.G]; tile += gridDim.x) {
        const int part = part_of_tile(tile_start, a.G, tile);
        int64_t begin, end;
        part_rows(a.offsets, a.n, part, begin, end);
        const float inv = 1.f / ((float)(end - begin) * (float)a.per_set);
        begin += (int64_t)(tile - tile_start[part]) * a.tile_rows;
        end = min(end, begin + a.tile_rows);
        const float* sums = a.sums + (int64_t)part * (2 * a.C + 1);
        __syncthreads();
        for (int s0 = 0; s0 < a.groups; s0 += sets_at_once) {
            const int set = s0 + threadIdx.x / L, l = threadIdx.x % L;
            float s1 = 0.f, s2 = 0.f;
            if (set < a.groups) {
                for (int c = set * a.per_set + l; c < (set + 1) * a.per_set; c += L) {
                    const float g = a.gamma ? __ldg(a.gamma + part * a.gamma_stride + c) : 1.f;
                    s1 += g * sums[c];
                    s2 += g * sums[a.C + c];
                }
            }
            s1 = lane_sum(s1, L);
            s2 = lane_sum(s2, L);
            if (set < a.groups && l == 0) of_set[set] = make_float2(s1 * inv, s2 * inv);
        }
        __syncthreads();
        // dx = rstd (gamma du - S1 / m) - (x - mean) rstd^2 S2 / m
        f2 minus_mean[4], scale[4], bet[4], m1[4], m2[4];
        {
            float rstd[8];
            load_coefficients(a, part, at, minus_mean, scale, bet, rstd);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 s0 = 2 * i < at.valid ? of_set[(8 * at.u + 2 * i) / a.per_set] : make_float2(0.f, 0.f);
                const float2 s1 = 2 * i + 1 < at.valid ? of_set[(8 * at.u + 2 * i + 1) / a.per_set] : make_float2(0.f, 0.f);
                m1[i] = pack2(-rstd[2 * i] * s0.x, -rstd[2 * i + 1] * s1.x);
                m2[i] = pack2(-rstd[2 * i] * rstd[2 * i] * s0.y, -rstd[2 * i + 1] * rstd[2 * i + 1] * s1.y);
            }
        }
        const float slope = a.slope ? __ldg(a.slope + part * a.slope_stride) : 0.f;
        if (at.active) {
            Eight<T> x[RB], d[RB];
            int64_t row = begin + at.y;
            int left = (int)(end - row), asked = left;
            const T* from = static_cast<const T*>(a.X) + row * a.ldx + 8 * at.u;
            const T* d_from = static_cast<const T*>(a.dY) + row * a.lddy + 8 * at.u;
            T* out = Y + row * a.ldy + 8 * at.u;
            const int64_t x_step = a.rows_at_once * a.ldx, d_step = a.rows_at_once * a.lddy, out_step = a.rows_at_once * a.ldy;
            auto request = [&](int b) {
                load_unit<FULL>(x[b], from, asked > 0, at.valid, a.vx);
                load_unit<FULL>(d[b], d_from, asked > 0, at.valid, a.vdy);
                from += x_step;
                d_from += d_step;
                asked -= a.rows_at_once;
            };
#pragma unroll
            for (int b = 0; b < RB; ++b) request(b);
            while (left > 0) {
#pragma unroll
                for (int b = 0; b < RB; ++b, row += a.rows_at_once, out += out_step) {
                    if (left <= 0) break;
                    left -= a.rows_at_once;
                    f2 t[4], du[4];
                    pairs_of(x[b], t);
                    pairs_of(d[b], du);
                    request(b);
                    back_centred(a, row, at.u, minus_mean, scale, bet, slope, t, du);
#pragma unroll
                    for (int i = 0; i < 4; ++i) du[i] = fma2(t[i], m2[i], fma2(du[i], scale[i], m1[i]));
                    store_unit<FULL>(out, du, at.valid, a.vy);
                }
            }
        }
    }
}

// The tiles' sums of every part added up in order: a block of 32 columns by 8 shares of the tiles.
__global__ void __launch_bounds__(NORM_THREADS) norm_reduce_kernel(const NormArgs a) {
    __shared__ int32_t tile_start[RTMA_MAX_GROUPS + 1], warp_sums[32];
    __shared__ float red[8][33];
    wait_for_kernel_before();
    number_tiles(a.offsets, a.n, a.G, a.tile_rows, a.tiles, tile_start, warp_sums);
    const int width = 2 * a.C + 1, lane = threadIdx.x & 31, share = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane, part = blockIdx.y;
    float s = 0.f;
    if (c < width)
        for (int t = tile_start[part] + share; t < tile_start[part + 1]; t += 8) s += a.partial[(int64_t)t * width + c];
    red[share][lane] = s;
    __syncthreads();
    if (share == 0 && c < width) {
        for (int k = 1; k < 8; ++k) s += red[k][lane];
        a.sums[(int64_t)part * width + c] = s;
        if (c < a.C) {
            if (a.dbeta && (a.dbeta_stride || a.G == 1)) a.dbeta[part * a.dbeta_stride + c] = s;
        } else if (c < 2 * a.C) {
            if (a.dgamma && (a.dgamma_stride || a.G == 1)) a.dgamma[part * a.dgamma_stride + c - a.C] = s;
        } else if (a.dslope && (a.dslope_stride || a.G == 1)) {
            a.dslope[part * a.dslope_stride] = s;
        }
    }
}

// Gradients of parameters that all parts share: the parts' sums added up in order.
__global__ void __launch_bounds__(NORM_THREADS) norm_reduce_parts_kernel(const NormArgs a) {
    wait_for_kernel_before();
    const int width = 2 * a.C + 1, c = blockIdx.x * NORM_THREADS + threadIdx.x;
    if (c >= width) return;
    float* to = c < a.C ? (a.dbeta && !a.dbeta_stride ? a.dbeta + c : nullptr)
                : c < 2 * a.C ? (a.dgamma && !a.dgamma_stride ? a.dgamma + c - a.C : nullptr)
                              : (a.dslope && !a.dslope_stride ? a.dslope : nullptr);
    if (!to) return;
    float s = 0.f;
    for (int g = 0; g < a.G; ++g) s += a.sums[(int64_t)g * width + c];
    *to = s;
}

template <class K>
K by_type(int32_t dtype, K f32, K bf16, K f16) { return dtype == RTMA_F32 ? f32 : dtype == RTMA_BF16 ? bf16 : f16; }
// of sets within units
#define NORM_KERNEL_WITHIN(name, full) (a.within == 1 ? NORM_KERNEL(name, , 1, full) : a.within == 2 ? NORM_KERNEL(name, , 2, full) : NORM_KERNEL(name, , 4, full))
#define NORM_KERNEL(name, ...) by_type(d->dtype, &name<float __VA_ARGS__>, &name<__nv_bfloat16 __VA_ARGS__>, &name<__half __VA_ARGS__>)

// Runs of rows, per_sm for every SM: twice as many as run at a time, so that all SMs end together.  A few rows per thread at least.
void cut_rows(NormArgs& a, const rtma_ctx* ctx, int per_sm) {
    const int64_t runs = (int64_t)per_sm * ctx->sm_count, least = 4 * (int64_t)a.rows_at_once, even = ceil_div(a.n, runs > 2 * a.G ? runs - a.G : a.G);
    a.tile_rows = (int)(even > least ? even : least);
    a.tiles = a.n / a.tile_rows + a.G;
}

// Whether every unit of eight channels is there in full, on the boundary of one load: then no load or store asks.
bool full_units(const NormArgs& a, int32_t dtype, bool gradient) {
    const int most = dtype == RTMA_F32 ? 32 : 16;
    const bool pieces = a.pitch == 0 || a.straddles || a.within || (a.units & (a.units - 1)) == 0;  // no lane of a row is idle, or the kernel asks
    return a.C % 8 == 0 && pieces && a.vx >= most && a.vy >= most && (!gradient || a.vdy >= most);
}

int32_t check_norm(rtma_ctx* ctx, const char* who, const rtma_norm_desc* d, int64_t n, int32_t G, const int64_t* offsets, const float* slope,
                   const float* stats) {
    if (!d) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: null descriptor", who);
    RTMA_TRY(check_parts(ctx, who, n, G, offsets));
    if (d->dtype < RTMA_F32 || d->dtype > RTMA_F16) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: dtype=%d", who, d->dtype);
    if (d->C < 1 || d->C > NORM_MAX_CHANNELS) return rtma_fail(ctx, RTMA_ERR_UNSUPPORTED, "%s: %d channels outside [1,%d]", who, d->C, NORM_MAX_CHANNELS);
    if (d->groups < 1 || d->C % d->groups) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: %d channels in %d sets", who, d->C, d->groups);
    if (d->scope != RTMA_SCOPE_ROW && d->scope != RTMA_SCOPE_PART) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: scope=%d", who, d->scope);
    if (d->act < RTMA_ACT_NONE || d->act > RTMA_ACT_SILU) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: act=%d", who, d->act);
    if (d->act == RTMA_ACT_PRELU && !slope) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: PReLU without a slope", who);
    if (!(d->eps > 0.f) || std::isinf(d->eps)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: eps=%g", who, (double)d->eps);
    if (!(d->p >= 0.0 && d->p <= 1.0)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: p=%g outside [0,1]", who, d->p);
    if (reinterpret_cast<uintptr_t>(stats) % sizeof(float2))  // (mean, 1 / std) are read and written as one
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: stats do not lie on an 8-byte boundary", who);
    return RTMA_OK;
}

NormArgs norm_args(const rtma_ctx* ctx, const rtma_norm_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx,
                   const float* gamma, const float* beta, const float* slope, const int32_t* row_ids) {
    NormArgs a{};
    a.offsets = offsets;
    a.n = n;
    a.G = G;
    a.C = d->C;
    a.groups = d->groups;
    a.per_set = d->C / d->groups;
    a.units = (d->C + 7) / 8;
    a.rows_at_once = NORM_THREADS / a.units;
    // warps keep rows to themselves where a set is a power of two of lanes or the whole row, or two sets at most share a unit
    const int lanes = a.per_set / 8;
    const bool of_lanes = d->groups == 1 || (a.per_set % 8 == 0 && (lanes & (lanes - 1)) == 0);
    a.straddles = !of_lanes && a.per_set >= 8;
    a.within = a.per_set == 1 || a.per_set == 2 || a.per_set == 4 ? a.per_set : 0;
    if (d->groups == 1) a.within = 0;
    if (d->scope == RTMA_SCOPE_ROW && (of_lanes || a.straddles || a.within))
        for (a.pitch = 1; a.pitch < a.units;) a.pitch *= 2;
    a.wide = a.pitch > 32 && (a.straddles || a.per_set > 256);
    cut_rows(a, ctx, 4);
    a.act = d->act;
    a.eps = d->eps;
    a.X = X;
    a.ldx = ldx;
    a.vx = row_granule(X, ldx, row_type_bytes(d->dtype));
    a.gamma = gamma;
    a.beta = beta;
    a.slope = d->act == RTMA_ACT_PRELU ? slope : nullptr;
    a.gamma_stride = d->gamma_stride;
    a.beta_stride = d->beta_stride;
    a.slope_stride = d->slope_stride;
    a.drop = drop_args(d->p, d->seed, row_ids);
    return a;
}

}  // namespace

extern "C" int32_t rtma_group_norm(rtma_ctx* ctx, const rtma_norm_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx,
                                   const float* gamma, const float* beta, const float* slope, const int32_t* row_ids, void* Y, int64_t ldy,
                                   float* stats, void* stream_) {
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_norm(ctx, "rtma_group_norm", d, n, G, offsets, slope, stats));
    if (n > 0 && (!X || !Y)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_group_norm: null pointer");
    if (ldx < d->C || ldy < d->C) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_group_norm: rows of %d channels lie closer than that", d->C);
    const bool rows = d->scope == RTMA_SCOPE_ROW;
    if (n == 0 && (rows || !stats)) return RTMA_OK;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    NormArgs a = norm_args(ctx, d, n, G, offsets, X, ldx, gamma, beta, slope, row_ids);
    a.Y = Y;
    a.ldy = ldy;
    a.vy = row_granule(Y, ldy, row_type_bytes(d->dtype));
    a.stats = stats;
    if (!rows) cut_rows(a, ctx, 6);
    const int64_t tiles = a.tiles;
    const size_t piece_bytes = rows ? 0 : ArenaCursor::granule(sizeof(float2) * tiles * a.groups);
    const size_t stat_bytes = rows || stats ? 0 : ArenaCursor::granule(sizeof(float2) * (size_t)G * a.groups);
    RTMA_TRY(prepare_row_call(ctx, piece_bytes + stat_bytes, stream));
    const unsigned grid = (unsigned)tiles;
    if (rows) {
        const size_t smem = sizeof(float) * a.rows_at_once * (8 * a.units + 2 * (size_t)a.groups);
        const bool full = full_units(a, d->dtype, false);
        auto kernel = !a.pitch ? NORM_KERNEL(norm_rows_kernel)
                      : a.within ? (full ? NORM_KERNEL_WITHIN(norm_unit_rows_kernel, true) : NORM_KERNEL_WITHIN(norm_unit_rows_kernel, false))
                      : a.straddles && a.wide ? (full ? NORM_KERNEL(norm_straddle_rows_kernel, , true, true) : NORM_KERNEL(norm_straddle_rows_kernel, , false, true))
                      : a.straddles ? (full ? NORM_KERNEL(norm_straddle_rows_kernel, , true, false) : NORM_KERNEL(norm_straddle_rows_kernel, , false, false))
                      : a.wide ? (full ? NORM_KERNEL(norm_warp_rows_kernel, , true, true) : NORM_KERNEL(norm_warp_rows_kernel, , false, true))
                               : (full ? NORM_KERNEL(norm_warp_rows_kernel, , true, false) : NORM_KERNEL(norm_warp_rows_kernel, , false, false));
        KernelScope ks(ctx, KC_POST, stream);
        launch_kernel(kernel, grid, NORM_THREADS, a.pitch ? 0 : smem, stream, a);
    } else {
        ArenaCursor cur(ctx->arena);
        a.pieces = cur.take<float2>(tiles * a.groups);
        if (!stats) a.stats = cur.take<float>(2 * (size_t)G * a.groups);
        if (n > 0) {
            KernelScope ks(ctx, KC_POST, stream);
            launch_kernel(full_units(a, d->dtype, false) ? NORM_KERNEL(norm_stats_kernel, , true) : NORM_KERNEL(norm_stats_kernel, , false), grid, NORM_THREADS, 0, stream, a);
        }
        RTMA_LAUNCH_CHECK(ctx);
        {
            KernelScope ks(ctx, KC_POST, stream);
            launch_kernel(norm_join_kernel, (unsigned)ceil_div((int64_t)G * a.groups * 32, NORM_THREADS), NORM_THREADS, 0, stream, a);
        }
        RTMA_LAUNCH_CHECK(ctx);
        if (n > 0) {
            KernelScope ks(ctx, KC_POST, stream);
            launch_kernel(full_units(a, d->dtype, false) ? NORM_KERNEL(norm_apply_kernel, , true) : NORM_KERNEL(norm_apply_kernel, , false), grid, NORM_THREADS, 0, stream, a);
        }
    }
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

extern "C" int32_t rtma_group_norm_grad(rtma_ctx* ctx, const rtma_norm_desc* d, int64_t n, int32_t G, const int64_t* offsets, const void* X, int64_t ldx,
                                        const void* dY, int64_t lddy, const float* stats, const float* gamma, const float* beta, const float* slope,
                                        const int32_t* row_ids, void* dX, int64_t lddx, float* dgamma, int64_t dgamma_stride, float* dbeta,
                                        int64_t dbeta_stride, float* dslope, int64_t dslope_stride, void* stream_) {
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    RTMA_TRY(check_norm(ctx, "rtma_group_norm_grad", d, n, G, offsets, slope, stats));
    if (n > 0 && (!X || !dY || !stats || !dX)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_group_norm_grad: null pointer");
    if (ldx < d->C || lddy < d->C || lddx < d->C)
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_group_norm_grad: rows of %d channels lie closer than that", d->C);
    const auto overlap = [&](const float* p, int64_t stride) { return p && G > 1 && stride != 0 && stride < d->C && stride > -d->C; };
    if (overlap(dgamma, dgamma_stride) || overlap(dbeta, dbeta_stride))
        return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_group_norm_grad: gradients of %d channels lie closer than that", d->C);
    if (dslope && d->act != RTMA_ACT_PRELU) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "rtma_group_norm_grad: a slope's gradient without PReLU");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    NormArgs a = norm_args(ctx, d, n, G, offsets, X, ldx, gamma, beta, slope, row_ids);
    a.dY = dY;
    a.lddy = lddy;
    a.vdy = row_granule(dY, lddy, row_type_bytes(d->dtype));
    a.Y = dX;
    a.ldy = lddx;
    a.vy = row_granule(dX, lddx, row_type_bytes(d->dtype));
    a.stats = const_cast<float*>(stats);
    a.dgamma = dgamma; a.dgamma_stride = dgamma_stride;
    a.dbeta = dbeta; a.dbeta_stride = dbeta_stride;
    a.dslope = dslope; a.dslope_stride = dslope_stride;
    const int64_t tiles = a.tiles, width = 2 * (int64_t)a.C + 1;
    RTMA_TRY(prepare_row_call(ctx, ArenaCursor::granule(sizeof(float) * tiles * width) + ArenaCursor::granule(sizeof(float) * G * width), stream));
    ArenaCursor cur(ctx->arena);
    a.partial = cur.take<float>(tiles * width);
    a.sums = cur.take<float>(G * width);
    const bool rows = d->scope == RTMA_SCOPE_ROW;
    if (n > 0) {
        KernelScope ks(ctx, KC_POST, stream);
        if (rows) {
            const size_t smem = sizeof(float2) * (8 * NORM_THREADS + (size_t)a.rows_at_once * a.groups);
            const bool full = full_units(a, d->dtype, true);
            auto kernel = !a.pitch ? NORM_KERNEL(norm_rows_grad_kernel)
                          : a.within ? (full ? NORM_KERNEL_WITHIN(norm_unit_rows_grad_kernel, true) : NORM_KERNEL_WITHIN(norm_unit_rows_grad_kernel, false))
                          : a.straddles && a.wide ? (full ? NORM_KERNEL(norm_straddle_rows_grad_kernel, , true, true) : NORM_KERNEL(norm_straddle_rows_grad_kernel, , false, true))
                          : a.straddles ? (full ? NORM_KERNEL(norm_straddle_rows_grad_kernel, , true, false) : NORM_KERNEL(norm_straddle_rows_grad_kernel, , false, false))
                          : a.wide ? (full ? NORM_KERNEL(norm_warp_rows_grad_kernel, , true, true) : NORM_KERNEL(norm_warp_rows_grad_kernel, , false, true))
                                   : (full ? NORM_KERNEL(norm_warp_rows_grad_kernel, , true, false) : NORM_KERNEL(norm_warp_rows_grad_kernel, , false, false));
            launch_kernel(kernel, (unsigned)tiles, NORM_THREADS, a.pitch ? 0 : smem, stream, a);
        } else {
            launch_kernel(full_units(a, d->dtype, true) ? NORM_KERNEL(norm_grad_sums_kernel, , true) : NORM_KERNEL(norm_grad_sums_kernel, , false), (unsigned)tiles, NORM_THREADS, 0, stream, a);
        }
    }
    RTMA_LAUNCH_CHECK(ctx);
    {
        KernelScope ks(ctx, KC_POST, stream);
        launch_kernel(norm_reduce_kernel, dim3((unsigned)ceil_div(width, 32), (unsigned)G), NORM_THREADS, 0, stream, a);
    }
    RTMA_LAUNCH_CHECK(ctx);
    if (G > 1 && ((dgamma && !dgamma_stride) || (dbeta && !dbeta_stride) || (dslope && !dslope_stride))) {
        KernelScope ks(ctx, KC_POST, stream);
        launch_kernel(norm_reduce_parts_kernel, (unsigned)ceil_div(width, NORM_THREADS), NORM_THREADS, 0, stream, a);
    }
    RTMA_LAUNCH_CHECK(ctx);
    if (n > 0 && !rows) {
        KernelScope ks(ctx, KC_POST, stream);
        launch_kernel(full_units(a, d->dtype, true) ? NORM_KERNEL(norm_grad_apply_kernel, , true) : NORM_KERNEL(norm_grad_apply_kernel, , false), (unsigned)tiles, NORM_THREADS, 0, stream, a);
    }
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}
