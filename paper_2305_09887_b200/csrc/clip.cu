// The norm of every part's gradients over all their tensors, and the gradients scaled down to a largest norm:
//   norm_g = sqrt(sum over the tensors of part g of sum x^2),  out = c_g x,  c_g = min(1, max_norm / norm_g)
//
// Two passes over the gradients.  Every tensor's share of a part is cut into pieces of equal length, of which a few thousand keep all SMs
// busy; the first pass leaves the sum of squares of every piece, the pieces of a part behind one another, and every block of the
// second adds up those of its part itself, always in the same order, so that no kernel lies between the two and no block waits for another.
// The second walks the pieces backwards: what the first has read last may still be in the L2 cache (fp32 in eight parts, 90 MB of gradients: 66 us, forwards 71;
// 180 MB 99, 101; 300 MB of bf16 into fp32 220 either way).
//
// Squares are added up in fp32 eight at a time, then in 64 bits; eight whose sum leaves the range of fp32 (or is so small that
// squares got lost) are squared in 64 bits.  So the norm neither overflows nor underflows before its own value does.
#include <algorithm>
#include <memory>
#include <new>
#include <utility>

#include "rows.cuh"

RTMA_BOUNDS_TU()

namespace {

constexpr int THREADS = 256, BLOCKS_PER_SM = 4;
constexpr int FEW = 24, MANY = 160;  // tensors that one launch takes, in its arguments

struct Tensor {
    const void* grad;
    void* out;
    int64_t size, grad_stride, out_stride;
    int32_t first;  // piece of a part at which the tensor starts
    int32_t types;  // grad's + 4 out's
};
template <int MOST>
struct ClipArgs {
    Tensor t[MOST];
    int count, G, per_part;    // per_part: pieces of a part in all launches
    int first, pieces;         // those of this launch
    int64_t length;            // of a piece
    double max_norm;
    bool zero_nonfinite, write_norms;
    bool one;                  // norm for all parts
    double* sums;              // [part][per_part]
    float* norms;
};

// A piece: the elements [begin, begin + length) of a tensor's share of a part.
struct Piece {
    int tensor;
    int64_t begin, length;
};
template <int MOST>
__device__ __forceinline__ Piece piece_of(const ClipArgs<MOST>& a, int r) {  // r: of this launch's pieces of a part
    int lo = 0, hi = a.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.t[mid].first <= r) lo = mid;
        else hi = mid;
    }
    const int64_t begin = (r - a.t[lo].first) * a.length;
    return {lo, begin, min(a.length, a.t[lo].size - begin)};
}

// The value of all threads' s in every thread; the order is fixed.
__device__ __forceinline__ double block_sum(double s, double* red) {
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    s = red[0];
#pragma unroll
    for (int k = 1; k < THREADS / 32; ++k) s += red[k];
    return s;
}

__device__ __forceinline__ double squares(const float (&v)[8]) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(v[j], v[j], s);
    if (s >= 1e-30f && s <= 1e37f) return s;
    double d = 0.0;  // (zeros, too)
#pragma unroll
    for (int j = 0; j < 8; ++j) d += (double)v[j] * v[j];
    return d;
}

// Eight values of a piece for a thread in a step: neighbouring ones where gradients and results lie on boundaries of eight values (VECTOR),
// otherwise every THREADS-th, so that a warp's are neighbours.  WHOLE: all of the step's values exist.
template <bool VECTOR, bool WHOLE, class T>
struct Step {
    Eight<T> e;
    T one[VECTOR ? 1 : 8];
    __device__ __forceinline__ void load(const T* p, int64_t length, int64_t step) {
        if constexpr (VECTOR) {
            const int64_t at = 8 * (step * THREADS + threadIdx.x);
            if constexpr (WHOLE) {
                load_unit<true>(e, p + at, true, 8, 32);
            } else {
                const int valid = (int)max((int64_t)0, min((int64_t)8, length - at));
                e.load(p + (valid ? at : 0), valid, 8 * (int)sizeof(T));
            }
        } else {
            const int64_t at = 8 * step * THREADS + threadIdx.x;
#pragma unroll
            for (int j = 0; j < 8; ++j) one[j] = WHOLE || at + j * THREADS < length ? p[at + j * THREADS] : from_f32<T>(0.f);
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if constexpr (VECTOR) {
            e.values(v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = to_f32(one[j]);
        }
    }
    // results are not read again here: they leave the L2 cache to the gradients
    template <class O>
    __device__ __forceinline__ static void store(O* p, int64_t length, int64_t step, const float (&v)[8]) {
        if constexpr (VECTOR) {
            const int64_t at = 8 * (step * THREADS + threadIdx.x);
            if constexpr (WHOLE) {
                if constexpr (sizeof(O) == 4) {  // whole sectors: two stores of 16 bytes each took 30 us more of the 250 for 151M bf16 values
                    asm volatile("st.global.cs.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + at), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]),
                                 "f"(v[7])
                                 : "memory");
                } else {
                    const O* tag = nullptr;
                    __stcs(reinterpret_cast<uint4*>(p + at), make_uint4(narrow2(v[0], v[1], tag), narrow2(v[2], v[3], tag), narrow2(v[4], v[5], tag), narrow2(v[6], v[7], tag)));
                }
            } else if (at < length) {
                store_eight(p + at, v, (int)min((int64_t)8, length - at), 8 * (int)sizeof(O));
            }
        } else {
            const int64_t at = 8 * step * THREADS + threadIdx.x;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (WHOLE || at + j * THREADS < length) p[at + j * THREADS] = from_f32<O>(v[j]);
        }
    }
};
// on a boundary of eight values
template <class T>
__device__ __forceinline__ bool on_eight(const T* p) { return (reinterpret_cast<uintptr_t>(p) & (8 * sizeof(T) - 1)) == 0; }

constexpr int TOGETHER = 4;  // steps of which all loads are under way at a time

template <bool VECTOR, class T>
__device__ __forceinline__ double piece_squares(const T* p, int64_t length) {
    double s = 0.0;
    const int64_t whole = length / (8 * THREADS);
    int64_t i = 0;
    float v[8];
    for (; i + TOGETHER <= whole; i += TOGETHER) {
        Step<VECTOR, true, T> step[TOGETHER];
#pragma unroll
        for (int k = 0; k < TOGETHER; ++k) step[k].load(p, length, i + k);
#pragma unroll
        for (int k = 0; k < TOGETHER; ++k) {
            step[k].values(v);
            s += squares(v);
        }
    }
    for (; i * 8 * THREADS < length; ++i) {
        Step<VECTOR, false, T> step;
        step.load(p, length, i);
        step.values(v);
        s += squares(v);
    }
    return s;
}

template <int MOST>
__global__ void __launch_bounds__(THREADS, BLOCKS_PER_SM) squares_kernel(const __grid_constant__ ClipArgs<MOST> a) {
    __shared__ double red[THREADS / 32];
    wait_for_kernel_before();
    const int64_t all = (int64_t)a.G * a.pieces;
    for (int64_t id = blockIdx.x; id < all; id += gridDim.x) {
        const int part = (int)(id / a.pieces), r = (int)(id - (int64_t)part * a.pieces);
        const Piece piece = piece_of(a, r);
        const Tensor& t = a.t[piece.tensor];
        const int64_t from = part * t.grad_stride + piece.begin;
        auto sum = [&](auto tag) {
            typedef decltype(tag) T;
            const T* p = static_cast<const T*>(t.grad) + from;
            return on_eight(p) ? piece_squares<true>(p, piece.length) : piece_squares<false>(p, piece.length);
        };
        const int type = t.types & 3;
        double s = type == RTMA_F32 ? sum(0.f) : type == RTMA_BF16 ? sum(__nv_bfloat16()) : sum(__half());
        s = block_sum(s, red);
        if (threadIdx.x == 0) a.sums[(int64_t)part * a.per_part + a.first + r] = s;
    }
}

// What the gradients of a part are multiplied by.
struct Scale {
    double norm, c;
    bool all, none;  // they stay as they are; they become zeros
};
template <int MOST>
__device__ __forceinline__ Scale scale_of(const ClipArgs<MOST>& a, int part, double* red) {
    const double* p = a.sums + (a.one ? 0 : (int64_t)part * a.per_part);
    const int count = a.one ? a.G * a.per_part : a.per_part;
    double s = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < count; i += THREADS) s += p[i];
    Scale x;
    x.norm = sqrt(block_sum(s, red));
    const bool finite = x.norm <= 1.7976931348623157e308;
    x.all = finite ? x.norm <= a.max_norm : !a.zero_nonfinite;
    x.none = !finite && a.zero_nonfinite;
    x.c = x.all ? 1.0 : x.none ? 0.0 : a.max_norm / x.norm;
    return x;
}

__device__ __forceinline__ void scale_eight(const Scale& x, float (&v)[8]) {
    if (x.all) return;
    const float c = (float)x.c;
    const bool tiny = x.c < 1e-30;  // of which fp32 has fewer bits, or none
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = x.none ? 0.f : tiny ? (float)(v[j] * x.c) : v[j] * c;
}

template <bool VECTOR, class T, class O>
__device__ __forceinline__ void piece_scaled(const T* p, O* out, int64_t length, const Scale& x) {
    const int64_t whole = length / (8 * THREADS);
    int64_t i = 0;
    float v[8];
    for (; i + TOGETHER <= whole; i += TOGETHER) {
        Step<VECTOR, true, T> step[TOGETHER];
#pragma unroll
        for (int k = 0; k < TOGETHER; ++k) step[k].load(p, length, i + k);
#pragma unroll
        for (int k = 0; k < TOGETHER; ++k) {
            step[k].values(v);
            scale_eight(x, v);
            step[k].store(out, length, i + k, v);
        }
    }
    for (; i * 8 * THREADS < length; ++i) {
        Step<VECTOR, false, T> step;
        step.load(p, length, i);
        step.values(v);
        scale_eight(x, v);
        step.store(out, length, i, v);
    }
}

template <int MOST>
__global__ void __launch_bounds__(THREADS, BLOCKS_PER_SM) scale_kernel(const __grid_constant__ ClipArgs<MOST> a) {
    __shared__ double red[THREADS / 32];
    wait_for_kernel_before();
    int held = -1;
    Scale x{};
    const int64_t all = (int64_t)a.G * a.pieces;
    for (int64_t back = blockIdx.x; back < all; back += gridDim.x) {
        const int64_t id = all - 1 - back;
        const int part = (int)(id / a.pieces), r = (int)(id - (int64_t)part * a.pieces);
        if (a.one ? held < 0 : part != held) {
            held = part;
            x = scale_of(a, part, red);
        }
        if (r == 0 && a.write_norms && threadIdx.x == 0 && (!a.one || part == 0)) a.norms[part] = (float)x.norm;
        const Piece piece = piece_of(a, r);
        const Tensor& t = a.t[piece.tensor];
        if (!t.out || (x.all && t.out == t.grad)) continue;
        const int64_t from = part * t.grad_stride + piece.begin, to = part * t.out_stride + piece.begin;
        auto scale = [&](auto tag, auto out_tag) {
            typedef decltype(tag) T;
            typedef decltype(out_tag) O;
            const T* p = static_cast<const T*>(t.grad) + from;
            O* out = static_cast<O*>(t.out) + to;
            if (on_eight(p) && on_eight(out)) piece_scaled<true>(p, out, piece.length, x);
            else piece_scaled<false>(p, out, piece.length, x);
        };
        const int type = t.types & 3;
        const bool wide = t.types >> 2 == RTMA_F32;
        if (type == RTMA_F32) scale(0.f, 0.f);
        else if (type == RTMA_BF16) wide ? scale(__nv_bfloat16(), 0.f) : scale(__nv_bfloat16(), __nv_bfloat16());
        else wide ? scale(__half(), 0.f) : scale(__half(), __half());
    }
}

template <int MOST>
__global__ void __launch_bounds__(THREADS) norms_kernel(const __grid_constant__ ClipArgs<MOST> a) {
    __shared__ double red[THREADS / 32];
    wait_for_kernel_before();
    const Scale x = scale_of(a, blockIdx.x, red);
    if (threadIdx.x == 0) a.norms[blockIdx.x] = (float)x.norm;
}

// All launches of one of the passes; each takes MOST tensors.
template <int MOST>
int32_t pass(rtma_ctx* ctx, const rtma_gradient* grads, int32_t count, bool second, ClipArgs<MOST>& a, cudaStream_t stream) {
    int32_t next = 0;
    a.first = 0;
    for (int32_t i = 0; i < count;) {
        a.count = a.pieces = 0;
        bool wanted = !second;
        const int32_t first = next;
        for (; i < count && a.count < MOST; ++i) {
            if (!grads[i].size) continue;
            Tensor& t = a.t[a.count++];
            t.grad = grads[i].grad;
            t.out = grads[i].out;
            t.size = grads[i].size;
            t.grad_stride = grads[i].grad_stride;
            t.out_stride = grads[i].out_stride;
            t.types = grads[i].dtype + 4 * grads[i].out_dtype;
            t.first = a.pieces;
            a.pieces += (int)ceil_div(t.size, a.length);
            wanted = wanted || t.out;
        }
        next += a.pieces;
        a.first = first;
        if (!a.count) break;
        a.write_norms = second && first == 0 && a.norms;
        if (!wanted && !a.write_norms) continue;
        const unsigned grid = (unsigned)std::min<int64_t>((int64_t)a.G * a.pieces, (int64_t)BLOCKS_PER_SM * ctx->sm_count);
        KernelScope ks(ctx, KC_REDUCE_SGD, stream);
        launch_kernel(second ? scale_kernel<MOST> : squares_kernel<MOST>, grid, THREADS, 0, stream, a);
        RTMA_LAUNCH_CHECK(ctx);
    }
    return RTMA_OK;
}

template <int MOST>
int32_t clip(rtma_ctx* ctx, const rtma_gradient* grads, int32_t count, int32_t G, bool one, int64_t length, int per_part, double max_norm, bool zero_nonfinite,
             float* norms, cudaStream_t stream) {
    ClipArgs<MOST> a{};
    a.G = G;
    a.one = one;
    a.per_part = per_part;
    a.length = length;
    a.max_norm = max_norm;
    a.zero_nonfinite = zero_nonfinite;
    a.sums = reinterpret_cast<double*>(ctx->arena);
    a.norms = norms;
    bool outs = false;
    for (int32_t i = 0; i < count; ++i) outs = outs || (grads[i].out && grads[i].size);
    RTMA_TRY(pass(ctx, grads, count, false, a, stream));
    if (outs) return pass(ctx, grads, count, true, a, stream);
    if (!norms) return RTMA_OK;
    KernelScope ks(ctx, KC_REDUCE_SGD, stream);
    launch_kernel(norms_kernel<MOST>, one ? 1u : (unsigned)G, THREADS, 0, stream, a);
    RTMA_LAUNCH_CHECK(ctx);
    return RTMA_OK;
}

// A result that is another's, or another's gradient, would be read after it has been written, or before.
int32_t check_results(rtma_ctx* ctx, const char* who, int32_t count, const rtma_gradient* grads) {
    typedef std::pair<const void*, int32_t> Place;
    Place few[2 * FEW];
    std::unique_ptr<Place[]> many;
    Place* places = few;
    if (count > FEW) {
        many.reset(new (std::nothrow) Place[2 * (size_t)count]);
        if (!(places = many.get())) return rtma_fail(ctx, RTMA_ERR_WORKSPACE, "%s: no host memory for %d gradients", who, count);
    }
    size_t used = 0;
    for (int32_t i = 0; i < count; ++i) {
        const rtma_gradient& t = grads[i];
        if (!t.out || !t.size) continue;
        places[used++] = Place(t.out, i);
        if (t.out != t.grad) places[used++] = Place(t.grad, -1);
    }
    std::sort(places, places + used);
    for (size_t k = 1; k < used; ++k)
        if (places[k].first == places[k - 1].first && places[k].second >= 0)
            return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: the result of gradient %d lies where another result or gradient does", who, places[k].second);
    return RTMA_OK;
}

}  // namespace

extern "C" int32_t rtma_clip_gradients(rtma_ctx* ctx, int32_t count, const rtma_gradient* grads, int32_t G, int32_t one_norm, double max_norm, int32_t zero_nonfinite,
                                       float* norms, void* stream_) {
    const char* who = "rtma_clip_gradients";
    if (!ctx) return RTMA_ERR_INVALID_ARG;
    if (count < 0 || (count > 0 && !grads)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: %d gradients", who, count);
    if (G < 1 || G > RTMA_MAX_GROUPS) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: G=%d outside [1,%d]", who, G, RTMA_MAX_GROUPS);
    if (!(max_norm >= 0.0)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: max_norm=%g", who, max_norm);
    double total = 0.0;
    for (int32_t i = 0; i < count; ++i) {
        const rtma_gradient& t = grads[i];
        if (t.dtype < RTMA_F32 || t.dtype > RTMA_F16 || (t.out && t.out_dtype != t.dtype && t.out_dtype != RTMA_F32))
            return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: gradient %d has type %d, its result %d", who, i, t.dtype, t.out_dtype);
        if (t.size < 0 || (t.size > 0 && !t.grad)) return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: gradient %d of %lld values", who, i, (long long)t.size);
        if (t.out && t.size && G > 1 && t.out_stride < t.size && t.out_stride > -t.size)
            return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: the parts of result %d overlap", who, i);
        if (t.out == t.grad && t.size && (t.out_dtype != t.dtype || (G > 1 && t.out_stride != t.grad_stride)))
            return rtma_fail(ctx, RTMA_ERR_INVALID_ARG, "%s: result %d lies on its gradient in another form", who, i);
        total += (double)t.size;
    }
    RTMA_TRY(check_results(ctx, who, count, grads));
    // Pieces: 24 for every SM or so, of 2,048 values or more (a step of a block)
    constexpr int64_t STEP = 8 * THREADS;
    if (total * G >= 9e15) return rtma_fail(ctx, RTMA_ERR_OVERFLOW, "%s: %g values", who, total * G);
    const int64_t length = STEP * std::max<int64_t>(1, (int64_t)(total * G / (24.0 * ctx->sm_count * STEP)));
    int64_t per_part = 0;
    for (int32_t i = 0; i < count; ++i) per_part += ceil_div(grads[i].size, length);
    if (per_part * G >= (int64_t(1) << 30)) return rtma_fail(ctx, RTMA_ERR_OVERFLOW, "%s: %lld tensors' parts", who, (long long)(per_part * G));
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    DeviceScope on(ctx->device);
    RTMA_CUDA(ctx, on.status);
    RTMA_TRY(prepare_row_call(ctx, sizeof(double) * (size_t)per_part * G, stream));
    return count <= FEW ? clip<FEW>(ctx, grads, count, G, one_norm != 0, length, (int)per_part, max_norm, zero_nonfinite != 0, norms, stream)
                        : clip<MANY>(ctx, grads, count, G, one_norm != 0, length, (int)per_part, max_norm, zero_nonfinite != 0, norms, stream);
}
