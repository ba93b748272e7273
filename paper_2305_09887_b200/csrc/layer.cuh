// What the kernels of whole layers share: products of rows whose results go through an activation, a gate or a residual branch on
// their way out (layer.cu: 16-bit rows, layer_split.cu: fp32 rows).
#pragma once

#include "activation.cuh"
#include "grouped_linear.cuh"

namespace grouped {

struct LayerArgs : LinearArgs {
    int width;            // columns of the result (of each of a gated layer's two matrices)
    int act;
    const float* slope;
    int64_t slope_stride;
    const void* side;     // rows read on the way out: the residual branch (or none), or the result's gradient
    int64_t lds;
    int gs;               // granule of these rows
    int g2;               // granule of the result's second half (gradient of a gated layer)
    float* slope_slots;   // gradient, PReLU: what every warp that drains a tile has of the slope's gradient, [tile][slope_warps]
    int slope_warps;
};

#ifdef __CUDACC__
// The bias of a warp's columns in shared memory: 32 at a time, `chunks` of them.  Held for as long as part and column stay.
struct LayerBias {
    float* at;  // 16-byte boundary
    int part = -1, n0 = -1;
    // column(i): where chunk i starts in the bias; edge(i): how many columns of it there are
    template <class T, class Column, class Edge>
    __device__ __forceinline__ void fetch(const LayerArgs& a, int of_part, int of_n0, int chunks, int lane, const T*, Column column, Edge edge) {
        if (of_part == part && of_n0 == n0) return;
        part = of_part;
        n0 = of_n0;
        const T* bias = static_cast<const T*>(a.bias) + part * a.bias_stride;
        __syncwarp();
        for (int i = 0; i < chunks; ++i) at[32 * i + lane] = lane < edge(i) ? to_f32(bias[column(i) + lane]) : 0.f;
        __syncwarp();
    }
    // eight of them, added to v
    __device__ __forceinline__ void add(f2 (&v)[4], int i, int q) const {
        const float4* b = reinterpret_cast<const float4*>(at + 32 * i + 8 * q);
        const float4 x = b[0], y = b[1];
        v[0] = add2(v[0], pack2(x.x, x.y));
        v[1] = add2(v[1], pack2(x.z, x.w));
        v[2] = add2(v[2], pack2(y.x, y.y));
        v[3] = add2(v[3], pack2(y.z, y.w));
    }
};

template <int Q>
__device__ __forceinline__ void eight_of(const float (&v)[32], f2 (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pack2(v[8 * Q + 2 * i], v[8 * Q + 2 * i + 1]);
}
template <int Q>
__device__ __forceinline__ void eight_to(const f2 (&x)[4], float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(x[i], v[8 * Q + 2 * i], v[8 * Q + 2 * i + 1]);
}
// Values from `valid` on become zero: tensor memory may hold anything in columns that are not the tile's, and a sum must not see it.
__device__ __forceinline__ void cut_eight(f2 (&x)[4], int valid) {
    if (valid >= 8) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        unpack2(x[i], a, b);
        x[i] = pack2(2 * i < valid ? a : 0.f, 2 * i + 1 < valid ? b : 0.f);
    }
}
#endif

}  // namespace grouped

// fp32 rows: the matrices are laid out in planes (scratch), the two of a gated layer by turns of 32 columns.
size_t layer_split_bytes(const grouped::LayerArgs& a, bool gated);
void describe_layer_split(grouped::LayerArgs& a, bool gated);  // tiles
int32_t launch_layer_split(rtma_ctx* ctx, grouped::LayerArgs& a, bool gated, bool gradient, void* planes, int cls, cudaStream_t stream);
