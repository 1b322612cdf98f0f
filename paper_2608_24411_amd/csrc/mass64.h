// mass64.h -- device helpers shared by the sampling kernels (sample.hip) and beam search's
// choice (beam.hip): values in scalar registers, and exponentials in fp64.
#pragma once

#include "common.h"

namespace {

// A value that all lanes hold, in scalar registers.
__device__ __forceinline__ float uniform(float v) {
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}
__device__ __forceinline__ double uniform(double v) {
    return __hiloint2double(__builtin_amdgcn_readfirstlane(__double2hiint(v)),
                            __builtin_amdgcn_readfirstlane(__double2loint(v)));
}

// 2^x in fp64 for x < 1023, zero up to -1023.  2^f = 1 + f g(f) on [-1/2, 1/2], g of degree 8
// interpolated at Chebyshev nodes: 3.7e-14 off at most, and exactly 1 at 0.  x + 1.5 2^52 has
// the whole number in its low bits, which go to the exponent: rounding, conversion and ldexp
// instructions in their place take 110 cycles a wave and element where this takes 80.  At
// -1023, where everything below is put, the exponent and the mantissa of 1 give zero.
__device__ __forceinline__ double exp2_64(double x) {
    x = fmax(x, -1023.0);
    const double t = x + 0x1.8p52, f = x - (t - 0x1.8p52);
    double p = 0x1.b63880a30e9ffp-24;
    p = fma(p, f, 0x1.63d136366db24p-20);
    p = fma(p, f, 0x1.ffcb9515a8016p-17);
    p = fma(p, f, 0x1.4308ac85aa947p-13);
    p = fma(p, f, 0x1.5d87fe86fe88ep-10);
    p = fma(p, f, 0x1.3b2ab7181b755p-7);
    p = fma(p, f, 0x1.c6b08d7047e52p-5);
    p = fma(p, f, 0x1.ebfbdff823cedp-3);
    p = fma(p, f, 0x1.62e42fefa39efp-1);
    p = fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + (int)((uint32_t)__double2loint(t) << 20), __double2loint(p));
}

}  // namespace
