// 2^x on the multiply-add units.
#pragma once

#include "draft.cuh"

namespace treekv {

// 2^x of a pair on the multiply-add units, for the share of the exponentials that the special-function unit would keep waiting:
// x = n + f with n the nearest integer (Cody and Waite's reduction, here without error) and 2^f by the polynomial of degree 5 with
// value 1 at 0 and the least largest relative error on [-1/2, 1/2] (found by Lawson's iteration; 1.7e-7 with its roundings, as much
// as the unit's own).  x stays below 128 (no larger result is made here; weights
// are at most about 1).  From 2^-127 down the result is 0; NaN stays NaN.
__device__ inline float2 exp2_fma(float2 x) {
    const float big = 12582912.f + 127.f;  // 1.5 * 2^23 + 127: adding it rounds to an integer, and n + 127 stands in the low bits
    asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x.x));  // -127
    asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x.y));
    const float2 one = make_float2(1.f, 1.f);
    const float2 t = fma2(x, one, make_float2(big, big)), n = fma2(t, one, make_float2(-big, -big)), f = fma2(n, make_float2(-1.f, -1.f), x);
    float2 p = make_float2(0x1.5bba14p-10f, 0x1.5bba14p-10f);
    p = fma2(p, f, make_float2(0x1.3cea88p-7f, 0x1.3cea88p-7f));
    p = fma2(p, f, make_float2(0x1.c6b752p-5f, 0x1.c6b752p-5f));
    p = fma2(p, f, make_float2(0x1.ebf9bcp-3f, 0x1.ebf9bcp-3f));
    p = fma2(p, f, make_float2(0x1.62e42ap-1f, 0x1.62e42ap-1f));
    p = fma2(p, f, one);
    return fma2(p, make_float2(__int_as_float(__float_as_int(t.x) << 23), __int_as_float(__float_as_int(t.y) << 23)), make_float2(0.f, 0.f));
}

}  // namespace treekv
