// fp32 values as operands of bf16 products.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>

#ifdef __CUDACC__
// Eight fp32 values as three bf16 numbers each, x = h + m + l exactly (but for bits below the smallest bf16 number).  h is cut off
// so that no finite value becomes an infinity, m is rounded to nearest so that the products left out (m l, l m, l l: below 2^-22 of
// the product) have no preferred sign.  An infinity or NaN leaves NaN in m.
__device__ __forceinline__ void split_eight(const uint32_t (&x)[8], uint4 (&planes)[3]) {
    uint32_t h[4], m[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = x[2 * i], b = x[2 * i + 1];
        h[i] = __byte_perm(a, b, 0x7632);
        const float r0 = __uint_as_float(a) - __uint_as_float(a & 0xFFFF0000u), r1 = __uint_as_float(b) - __uint_as_float(b & 0xFFFF0000u);
        const __nv_bfloat162 t = __floats2bfloat162_rn(r0, r1);
        m[i] = *reinterpret_cast<const uint32_t*>(&t);
        l[i] = __byte_perm(__float_as_uint(r0 - __uint_as_float(m[i] << 16)), __float_as_uint(r1 - __uint_as_float(m[i] & 0xFFFF0000u)), 0x7632);
    }
    planes[0] = make_uint4(h[0], h[1], h[2], h[3]);
    planes[1] = make_uint4(m[0], m[1], m[2], m[3]);
    planes[2] = make_uint4(l[0], l[1], l[2], l[3]);
}
#endif
