// Numbers as unevaluated sums of two float32 (some 46 bits), where float64 would be
// waited for: it runs at 1/64 of float32's rate here, and a chain of its operations takes
// longer than ten float32 ones each.  Sums and products after Dekker (1971) and Knuth's
// two-sum; sines and cosines by their Taylor series.
#pragma once
#include <cuda_runtime.h>

namespace aces {

struct Two {
    float h, l;  // l at most half a unit of h
};
__device__ __forceinline__ Two two_sum(float a, float b) {
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two two_near(float a, float b) {  // |a| >= |b|
    const float s = __fadd_rn(a, b);
    return {s, __fsub_rn(b, __fsub_rn(s, a))};
}
__device__ __forceinline__ Two two_product(float a, float b) {  // exact
    const float p = __fmul_rn(a, b);
    return {p, __fmaf_rn(a, b, -p)};
}
__device__ __forceinline__ Two operator+(Two a, Two b) {
    Two s = two_sum(a.h, b.h);
    const Two t = two_sum(a.l, b.l);
    s = two_near(s.h, __fadd_rn(s.l, t.h));
    return two_near(s.h, __fadd_rn(s.l, t.l));
}
__device__ __forceinline__ Two operator-(Two a) { return {-a.h, -a.l}; }
__device__ __forceinline__ Two operator*(Two a, Two b) {
    const Two p = two_product(a.h, b.h);
    return two_near(p.h, __fmaf_rn(a.h, b.l, __fmaf_rn(a.l, b.h, p.l)));
}
__host__ __device__ constexpr Two two_of(double x) { return {(float)x, (float)(x - (double)(float)x)}; }

// 1 / sqrt(m): the estimate r and (1 - m r^2) of it
__device__ __forceinline__ Two two_rsqrt(Two m) {
    const float r = rsqrtf(m.h);
    const Two e = Two{1.0f, 0.0f} + -(m * two_product(r, r));
    return two_near(r, __fmul_rn(__fmul_rn(r, e.h), __fmaf_rn(0.375f, e.h, 0.5f)));
}

// sine and cosine of t turns, |t| <= 1/2
__device__ __forceinline__ void two_sincos(Two t, Two &sn, Two &cn) {
    const float q = rintf(4.0f * t.h);  // quarters
    const Two r = two_near(__fmaf_rn(-0.25f, q, t.h), t.l);
    const Two x = r * two_of(6.283185307179586) + Two{__fmul_rn(r.h, 2.4492935982947064e-16f), 0.0f}, z = x * x;
    // sin x = x + x z (-1/6 + z (1/120 - z (1/5040 - ...))), below pi / 4
    const float hs = __fmaf_rn(z.h, __fmaf_rn(z.h, __fmaf_rn(z.h, -1.0f / 1307674368000.0f, 1.0f / 6227020800.0f), -1.0f / 39916800.0f), 1.0f / 362880.0f);
    Two s = two_of(-1.0 / 5040) + two_product(z.h, hs);
    s = two_of(1.0 / 120) + z * s;
    s = two_of(-1.0 / 6) + z * s;
    s = x + x * (z * s);
    // cos x = 1 - z / 2 + z^2 (1/24 - z (1/720 - ...))
    const float hc = __fmaf_rn(z.h, __fmaf_rn(z.h, -1.0f / 87178291200.0f, 1.0f / 479001600.0f), -1.0f / 3628800.0f);
    Two c = two_of(1.0 / 40320) + two_product(z.h, hc);
    c = two_of(-1.0 / 720) + z * c;
    c = two_of(1.0 / 24) + z * c;
    c = two_of(-0.5) + z * c;
    c = Two{1.0f, 0.0f} + z * c;
    const int k = (int)q & 3;
    sn = k == 0 ? s : k == 1 ? c : k == 2 ? -s : -c;
    cn = k == 0 ? c : k == 1 ? -s : k == 2 ? -c : s;
}

}  // namespace aces
