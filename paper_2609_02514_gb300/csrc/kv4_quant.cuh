// Numbers to the codes of a 4-bit cache row (the format: kv4.cuh), a group a thread.
#pragma once
#include "kv4.cuh"

namespace aces {

// D / 8 numbers -> D / 64 words of codes and the group's t
template <int G, bool F32>
__device__ __forceinline__ void quantise(float (&x)[G], uint32_t (&w)[G / 8], float *t_out, bool *bad) {
    // the largest and the smallest, three at a time; NaN when there is one
    float mx = x[0], mn = x[0];
#pragma unroll
    for (int i = 1; i < G; i += 2) {
        const float y = x[i], z = x[i + 1 < G ? i + 1 : i];
        asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(mx) : "f"(y), "f"(z));
        asm("min.NaN.f32 %0, %0, %1, %2;" : "+f"(mn) : "f"(y), "f"(z));
    }
    *bad = false;
    if (!(mx <= KV4_CAP && mn >= -KV4_CAP)) {
        mx = -KV4_CAP, mn = KV4_CAP;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            *bad |= !(fabsf(x[i]) <= FLT_MAX);
            x[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -KV4_CAP), KV4_CAP) : 0.0f;
            mx = fmaxf(mx, x[i]), mn = fminf(mn, x[i]);
        }
    }
    float a = mx > -mn ? mx : mn;
    if (mx == -mn) {  // of both signs: the first
#pragma unroll
        for (int i = G - 1; i >= 0; --i)
            if (fabsf(x[i]) == mx) a = x[i];
    }
    const float t = kv4_t(a), s = t * KV4_STEP;
    const float inv = s == 0.0f ? 0.0f : __frcp_rn(s), h = s == 0.0f ? INFINITY : 0.5f * fabsf(s);
#pragma unroll
    for (int i = 0; i < G / 8; ++i) {
        w[i] = KV4_BITS;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[i] += kv4_round<F32>(x[8 * i + e], s, inv, h) << (4 * (e >> 1) + 16 * (e & 1));
    }
    *t_out = t;
}

}  // namespace aces
