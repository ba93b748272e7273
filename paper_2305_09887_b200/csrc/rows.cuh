// Shared by the operators on rows that are stored part after part (dropout, group norm, grouped products): element types, eight
// values of a row at a time, the walk over tiles that never straddle two parts, the dropout mask, and the host checks they have
// in common.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "common.cuh"

// ---- host ---------------------------------------------------------------------------------------
// Makes the context's device current for the length of a call.
struct DeviceScope {
    int before = -1;
    cudaError_t status;
    explicit DeviceScope(int device) {
        status = cudaGetDevice(&before);
        if (status == cudaSuccess && before != device) status = cudaSetDevice(device);
        else before = -1;
    }
    ~DeviceScope() {
        if (before >= 0) cudaSetDevice(before);
    }
};

inline size_t row_type_bytes(int32_t dtype) { return dtype == RTMA_F32 ? 4 : 2; }
// The largest power of two, up to 32 bytes, on whose multiples all rows lie.
inline int row_granule(const void* p, int64_t ld, size_t element) {
    const uintptr_t both = reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * (int64_t)element) | 32;
    return (int)(both & (~both + 1));
}
// Whether `stream` is being captured into a graph: such a call neither grows the scratch nor waits for other streams.
int32_t stream_captures(rtma_ctx* ctx, cudaStream_t stream, bool* captures);
// Scratch of a row operator's call on `stream`: grows it (not inside a capture), keeps a captured one alive, orders the call
// behind the last training call's streams.
int32_t prepare_row_call(rtma_ctx* ctx, size_t scratch_bytes, cudaStream_t stream);
// offsets, row count and number of parts as every row operator takes them
int32_t check_parts(rtma_ctx* ctx, const char* who, int64_t n, int32_t G, const int64_t* offsets);

// Dropout: the threshold of the 16-bit lanes and what kept values are multiplied by.
struct DropArgs {
    uint64_t base = 0;       // one SplitMix64 step of the seed
    uint32_t threshold = 0;  // of 65536: lanes below it are dropped; 0: no dropout
    float scale = 1.f;
    const int32_t* ids = nullptr;  // ids of the rows, or the rows' own numbers
};
inline uint64_t splitmix64_host(uint64_t z) {
    z += 0x9E3779B97F4A7C15ULL;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ULL;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBULL;
    return z ^ (z >> 31);
}
inline DropArgs drop_args(double p, uint64_t seed, const int32_t* ids) {
    DropArgs d;
    d.base = splitmix64_host(seed);
    d.threshold = (uint32_t)std::floor(65536.0 * p + 0.5);
    d.scale = d.threshold < 65536u ? (float)(65536.0 / (double)(65536u - d.threshold)) : 0.f;
    d.ids = ids;
    return d;
}

#ifdef __CUDACC__
// ---- eight values of a row ------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ void widen2(uint32_t w, float& a, float& b, const __nv_bfloat16*) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ void widen2(uint32_t w, float& a, float& b, const __half*) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
}
__device__ __forceinline__ uint32_t narrow2(float a, float b, const __nv_bfloat16*) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ uint32_t narrow2(float a, float b, const __half*) {
    const __half2 t = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}

// Eight consecutive values as they are stored; `valid` of them exist (the others read as zero).  p lies on a multiple of
// `granule` bytes.
template <class T>
struct Eight {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p, int valid, int granule) {
        uint32_t* q = reinterpret_cast<uint32_t*>(w);
        constexpr int WORDS = 2 * sizeof(T);
        if (sizeof(T) == 4 && valid == 8 && granule == 32) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]), "=r"(q[WORDS - 4]), "=r"(q[WORDS - 3]), "=r"(q[WORDS - 2]), "=r"(q[WORDS - 1])
                         : "l"(p));
        } else if (valid == 8 && granule >= 16) {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
        } else if (granule >= 8 && valid % (8 / (int)sizeof(T)) == 0) {
            // By pieces that are there or not: nothing is put together from loaded values, so that nothing waits for them here (which
            // tails by single 16-bit values do: they made the rows of a warp wait for one another's).
#pragma unroll
            for (int i = 0; i < WORDS / 2; ++i) {
                uint2 x = make_uint2(0u, 0u);
                if ((i + 1) * (8 / (int)sizeof(T)) <= valid) x = reinterpret_cast<const uint2*>(p)[i];
                q[2 * i] = x.x;
                q[2 * i + 1] = x.y;
            }
        } else if (granule >= 4 && valid % (4 / (int)sizeof(T)) == 0) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) q[i] = (i + 1) * (4 / (int)sizeof(T)) <= valid ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
        } else if constexpr (sizeof(T) == 2) {
            T e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j < valid ? p[j] : from_f32<T>(0.f);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                q[j] = (uint32_t)*reinterpret_cast<const unsigned short*>(&e[2 * j]) | (uint32_t)*reinterpret_cast<const unsigned short*>(&e[2 * j + 1]) << 16;
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        const uint32_t* q = reinterpret_cast<const uint32_t*>(w);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(q[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) widen2(q[j], v[2 * j], v[2 * j + 1], static_cast<const T*>(nullptr));
        }
    }
};
// FULL: all eight exist and lie on 16 bytes (fp32: 32); then one instruction, and none for rows that are not there.
template <bool FULL, class T>
__device__ __forceinline__ void load_unit(Eight<T>& e, const T* p, bool here, int valid, int granule) {
    if constexpr (FULL) {
        if (!here) {
#pragma unroll
            for (int i = 0; i < (int)(sizeof(T) / 2); ++i) e.w[i] = make_uint4(0u, 0u, 0u, 0u);
        } else if constexpr (sizeof(T) == 4) {
            uint32_t* q = reinterpret_cast<uint32_t*>(e.w);
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]), "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7])
                         : "l"(p));
        } else {
            e.w[0] = *reinterpret_cast<const uint4*>(p);
        }
    } else {
        e.load(p, here ? valid : 0, granule);
    }
}

template <class T>
__device__ __forceinline__ void store_eight(T* p, const float (&v)[8], int valid, int granule) {
    constexpr int WORDS = 2 * sizeof(T);
    uint32_t q[WORDS];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = __float_as_uint(v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = narrow2(v[2 * j], v[2 * j + 1], static_cast<const T*>(nullptr));
    }
    if (sizeof(T) == 4 && valid == 8 && granule == 32) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(q[0]), "r"(q[1]), "r"(q[2]), "r"(q[3]),
                     "r"(q[WORDS - 4]), "r"(q[WORDS - 3]), "r"(q[WORDS - 2]), "r"(q[WORDS - 1])
                     : "memory");
    } else if (valid == 8 && granule >= 16) {
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]);
    } else if (granule >= 8 && valid % (8 / (int)sizeof(T)) == 0) {
#pragma unroll
        for (int i = 0; i < WORDS / 2; ++i)
            if ((i + 1) * (8 / (int)sizeof(T)) <= valid) reinterpret_cast<uint2*>(p)[i] = make_uint2(q[2 * i], q[2 * i + 1]);
    } else if (granule >= 4 && valid % (4 / (int)sizeof(T)) == 0) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            if ((i + 1) * (4 / (int)sizeof(T)) <= valid) reinterpret_cast<uint32_t*>(p)[i] = q[i];
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < valid) reinterpret_cast<unsigned short*>(p)[j] = (unsigned short)(j & 1 ? q[j >> 1] >> 16 : q[j >> 1]);
    }
}

// ---- two fp32 numbers per instruction -------------------------------------------------------------
typedef unsigned long long f2;  // the lower half first
__device__ __forceinline__ f2 pack2(float a, float b) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float halves_sum(f2 x) {
    float a, b;
    unpack2(x, a, b);
    return a + b;
}

// Eight values as four pairs.
template <class T>
__device__ __forceinline__ void pairs_of(const Eight<T>& e, f2 (&v)[4]) {
    float x[8];
    e.values(x);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2(x[2 * i], x[2 * i + 1]);
}
template <bool FULL, class T>
__device__ __forceinline__ void store_unit(T* p, const f2 (&v)[4], int valid, int granule) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(v[i], x[2 * i], x[2 * i + 1]);
    store_eight(p, x, FULL ? 8 : valid, FULL ? (sizeof(T) == 4 ? 32 : 16) : granule);
}
template <class T>
__device__ __forceinline__ void store_pairs(T* p, const f2 (&v)[4], int valid, int granule) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(v[i], x[2 * i], x[2 * i + 1]);
    store_eight(p, x, valid, granule);
}

// ---- parts ----------------------------------------------------------------------------------------
// Rows of part g: [offsets[g], offsets[g + 1]) cut to [0, n), so that offsets that are no offsets reach no memory outside the
// rows.  offsets == NULL: one part of all rows.  span: that many parts as one.
__device__ __forceinline__ void part_rows(const int64_t* offsets, int64_t n, int g, int64_t& begin, int64_t& end, int span = 1) {
    if (!offsets) {
        begin = 0;
        end = n;
        return;
    }
    const int64_t a = __ldg(offsets + g), b = __ldg(offsets + g + span);
    if (!rtma_index_ok(a, n + 1, 8) || !rtma_index_ok(b - a, n + 1, 8)) {
        begin = end = 0;
        return;
    }
    begin = a < 0 ? 0 : (a > n ? n : a);
    end = b < begin ? begin : (b > n ? n : b);
}

// tile_start[g] = tiles of `tile_rows` rows in the parts before g, for g = 0..G, `limit` at most (which parts that follow one
// another never pass); every thread of a block takes part.
__device__ __forceinline__ void number_tiles(const int64_t* offsets, int64_t n, int G, int64_t tile_rows, int64_t limit, int32_t* tile_start,
                                             int32_t* warp_sums, int span = 1) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int64_t carry = 0;
    for (int base = 0; base < G; base += blockDim.x) {
        const int g = base + threadIdx.x;
        int32_t mine = 0;
        if (g < G) {
            int64_t a, b;
            part_rows(offsets, n, g, a, b, span);
            mine = (int32_t)((b - a + tile_rows - 1) / tile_rows);
        }
        int64_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t t = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += t;
        }
        if (lane == 31) warp_sums[warp] = (int32_t)min(upto, limit);
        __syncthreads();
        int64_t before = carry, total = carry;
        for (int w = 0; w < warps; ++w) {
            if (w < warp) before += warp_sums[w];
            total += warp_sums[w];
        }
        if (g < G) tile_start[g] = (int32_t)min(before + upto - mine, limit);
        carry = total;
        __syncthreads();
    }
    if (threadIdx.x == 0) tile_start[G] = (int32_t)min(carry, limit);
    __syncthreads();
}

// The part that a tile lies in (tile < tile_start[G]).
__device__ __forceinline__ int part_of_tile(const int32_t* tile_start, int G, int tile) {
    int lo = 0, hi = G;  // tile_start[lo] <= tile < tile_start[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tile_start[mid] <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

// ---- dropout --------------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t splitmix64(uint64_t z) {
    z += 0x9E3779B97F4A7C15ULL;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ULL;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBULL;
    return z ^ (z >> 31);
}
// v[j] *= 0 or scale for columns 8 unit .. 8 unit + 7 of the row with this id.  One 64-bit word decides over four columns, 16
// bits each; dropped values become +0 whatever they were.
__device__ __forceinline__ void drop_eight(const DropArgs& d, uint32_t id, uint32_t unit, float (&v)[8]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const uint64_t word = splitmix64(d.base ^ ((uint64_t)id << 32 | (2 * unit + q)));
        const uint32_t lo = (uint32_t)word, hi = (uint32_t)(word >> 32);
        v[4 * q + 0] = (lo & 0xFFFFu) >= d.threshold ? v[4 * q + 0] * d.scale : 0.f;
        v[4 * q + 1] = (lo >> 16) >= d.threshold ? v[4 * q + 1] * d.scale : 0.f;
        v[4 * q + 2] = (hi & 0xFFFFu) >= d.threshold ? v[4 * q + 2] * d.scale : 0.f;
        v[4 * q + 3] = (hi >> 16) >= d.threshold ? v[4 * q + 3] * d.scale : 0.f;
    }
}
__device__ __forceinline__ void drop_pairs(const DropArgs& d, uint32_t id, uint32_t unit, f2 (&v)[4]) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(v[i], x[2 * i], x[2 * i + 1]);
    drop_eight(d, id, unit, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2(x[2 * i], x[2 * i + 1]);
}
#endif
