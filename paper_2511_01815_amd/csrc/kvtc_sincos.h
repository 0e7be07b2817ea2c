// Sine and cosine of angles in double precision, for the rotations of keys and queries.  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kvtc {

// sin and cos of an angle of at most 2^31: what is left of it beyond the nearest multiple of pi/2 -- taken off in three parts with fused operations (Cody and Waite's
// reduction), to 2^-53 -- by the series about 0, to its 17th and 16th power.  (At pi/4 the next terms are r^19 / 19! = 2^-63.4 and r^18 / 18! = 2^-58.8, below half a last place.)
__device__ __forceinline__ void sincos_reduced(double angle, double* s, double* c) {
    const double n = __builtin_rint(angle * 0.63661977236758134308);                 // 2 / pi
    double r = __builtin_fma(n, -1.5707963267948966, angle);
    r = __builtin_fma(n, -6.123233995736766e-17, r);
    r = __builtin_fma(n, 1.4973849048591833e-33, r);
    const double q = r * r;
    double u = 1.0 / 355687428096000.0, v = 1.0 / 20922789888000.0;                  // 17!, 16!
    u = __builtin_fma(u, q, -1.0 / 1307674368000.0);
    v = __builtin_fma(v, q, -1.0 / 87178291200.0);
    u = __builtin_fma(u, q, 1.0 / 6227020800.0);
    v = __builtin_fma(v, q, 1.0 / 479001600.0);
    u = __builtin_fma(u, q, -1.0 / 39916800.0);
    v = __builtin_fma(v, q, -1.0 / 3628800.0);
    u = __builtin_fma(u, q, 1.0 / 362880.0);
    v = __builtin_fma(v, q, 1.0 / 40320.0);
    u = __builtin_fma(u, q, -1.0 / 5040.0);
    v = __builtin_fma(v, q, -1.0 / 720.0);
    u = __builtin_fma(u, q, 1.0 / 120.0);
    v = __builtin_fma(v, q, 1.0 / 24.0);
    u = __builtin_fma(u, q, -1.0 / 6.0);
    v = __builtin_fma(v, q, -0.5);
    u = __builtin_fma(u * q, r, r);
    v = __builtin_fma(v, q, 1.0);
    const uint32_t k = (uint32_t)(int32_t)n;
    const double a = k & 1u ? v : u, b = k & 1u ? u : v;
    *s = k & 2u ? -a : a;
    *c = (k + 1u) & 2u ? -b : b;
}

}  // namespace kvtc
