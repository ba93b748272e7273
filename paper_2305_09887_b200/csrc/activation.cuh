// The activations behind a norm or a product, eight values at a time, and their derivatives.
#pragma once

#include "rows.cuh"

#ifdef __CUDACC__
// 1 / (1 + exp(-u)): two special-function instructions, relative error a few 2^-23 (1 + |u|)
__device__ __forceinline__ f2 sigmoid2(f2 u) {
    const float log2e = 1.4426950408889634f;
    float a, b;
    unpack2(mul2(u, pack2(-log2e, -log2e)), a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    unpack2(add2(pack2(a, b), pack2(1.f, 1.f)), a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return pack2(a, b);
}

__device__ __forceinline__ void activate(int act, float slope, f2 (&u)[4]) {
    if (act == RTMA_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = mul2(u[i], sigmoid2(u[i]));
    } else if (act == RTMA_ACT_RELU) {  // NaN stays NaN
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a, b;
            unpack2(u[i], a, b);
            asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(a));
            asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(b));
            u[i] = pack2(a, b);
        }
    } else if (act == RTMA_ACT_PRELU) {
        const f2 slopes = pack2(slope, slope);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a, b, x, y;
            unpack2(u[i], a, b);
            unpack2(mul2(u[i], slopes), x, y);
            u[i] = pack2(a > 0.f ? a : x, b > 0.f ? b : y);
        }
    }
}
// d (holding dh) becomes du; returns the slope's gradient
__device__ __forceinline__ float activate_back(int act, float slope, const f2 (&u)[4], f2 (&d)[4]) {
    float ds = 0.f;
    if (act == RTMA_ACT_SILU) {
        const f2 one = pack2(1.f, 1.f), minus = pack2(-1.f, -1.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f2 g = sigmoid2(u[i]);
            d[i] = mul2(d[i], mul2(g, fma2(u[i], fma2(g, minus, one), one)));
        }
    } else if (act == RTMA_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a, b, x, y;
            unpack2(u[i], a, b);
            unpack2(d[i], x, y);
            d[i] = pack2(a > 0.f ? x : 0.f, b > 0.f ? y : 0.f);
        }
    } else if (act == RTMA_ACT_PRELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a, b, x, y;
            unpack2(u[i], a, b);
            unpack2(d[i], x, y);
            ds = fmaf(x, a > 0.f ? 0.f : a, ds);
            ds = fmaf(y, b > 0.f ? 0.f : b, ds);
            d[i] = pack2(a > 0.f ? x : x * slope, b > 0.f ? y : y * slope);
        }
    }
    return ds;
}

// The gate of a gated layer: from g, u and dh (the gradient of h = act(g) u) those of g and of u; returns the slope's gradient.
__device__ __forceinline__ float gate_back(int act, float slope, const f2 (&g)[4], const f2 (&u)[4], const f2 (&dh)[4], f2 (&dg)[4], f2 (&du)[4]) {
    float ds = 0.f;
    if (act == RTMA_ACT_SILU) {
        const f2 one = pack2(1.f, 1.f), minus = pack2(-1.f, -1.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f2 s = sigmoid2(g[i]);
            du[i] = mul2(dh[i], mul2(g[i], s));
            dg[i] = mul2(mul2(dh[i], u[i]), mul2(s, fma2(g[i], fma2(s, minus, one), one)));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            dg[i] = mul2(dh[i], u[i]);
            du[i] = g[i];
        }
        activate(act, slope, du);
#pragma unroll
        for (int i = 0; i < 4; ++i) du[i] = mul2(dh[i], du[i]);
        ds = activate_back(act, slope, g, dg);
    }
    return ds;
}
#endif
