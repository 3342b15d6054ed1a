// Rotation of queries and keys by their positions, with their norms, and the write of
// the keys so made and of the values into a 4-bit cache (the format: kv4.cuh).
//
//   y = x w / sqrt(mean(x^2) + eps)           (a head's D numbers; without norms y = x)
//   z_u = y_u c_j - y_v s_j, z_v = y_v c_j + y_u s_j     c_j, s_j = scale (cos, sin)(p f_j)
//
// for the pairs j < R / 2 of channels (u, v) = (j, j + R / 2), or (2 j, 2 j + 1); p is the
// position on the pair's axis.  As many warps as fit take the tokens in turns, one (or
// some, where there are few heads) at a time, and wait for nobody; a token's cosines and
// sines are made once, into shared memory.  A lane has both channels of its pairs, so no
// number changes lanes:
//   - of rows that stay numbers 16 channels, eight or four lanes a row, each with every
//     so many 16 bytes of it (a load or store of the warp covers whole sectors) and with
//     its weights, cosines and sines in registers for all heads;
//   - of rows that go to the cache two whole groups, four lanes a row, to be quantised.
//
// The angle p f is taken as turns, a 64-bit fraction f / (2 pi) times p (a position of 2^20
// has no fraction left in float32): whole turns fall off by themselves.  Beyond 2^26 the
// rounding of p f as a product in 64 bits comes to show, and is added.
//
// The cache's codes are those of z in 64 bits, so that they do not depend on how sums and
// products were ordered here.  Float32's z is within E of that; where a quotient lies
// closer than that to a border, or the step could be another, the whole warp does the
// row again to 46 bits (three rows of a thousand), or in float64 where those do not decide
// or products could pass float32.
//
// What bounds it.  Rotation of 8192 tokens of two sequences, 32 and 8 heads of 128 in
// bfloat16 (336 MB): 59 us, 5.7 TB/s; a copy of as many dense bytes takes 52.  Bytes under way
// are what counts: through registers, which hold two steps, it was 66 whatever the number of
// warps or instructions, and with a pipeline that ran dry behind every token; four steps of
// 1 KB a warp through shared memory, across tokens, are enough (six: 59).
// Into the cache, 80 tokens of 64 sequences: 43 us (111 MB), 35 when no row is done again: a
// warp that meets one is late by some 9 us, and has two or three tokens in all.  In
// float64 those rows made it 48, one after another by their four lanes 94.
#define ACES_FILE 10  // site numbers of the checked build
#include <climits>

#include "kv4_quant.cuh"
#include "turn.cuh"
#include "twofold.cuh"

namespace aces {

constexpr int TW = 4, TN = TW * 32;
constexpr int TOKENS = 8;  // of a warp, at most
// A unit's rows go to several warps while there are fewer units than this for an SM (image
// tokens, 4611 of 12 and 4 heads of 64 in float32: with 24 12.4 us, with 36 15.5; with 0 one
// token of 32 and 8 heads 10.5 us instead of 8).
constexpr long long SLICE_WARPS = 24;

// ---------------------------------------------------------------------------
// loads and stores
// (in place, a row is read by the lanes that write it, before they do: a plain load)
__device__ __forceinline__ uint4 load16(const void *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// 16 bytes of a row: its numbers, whatever the alignment
template <bool VEC, bool F32>
__device__ __forceinline__ uint4 load_word(const void *base, int at) {  // at: in numbers
    const char *p = reinterpret_cast<const char *>(base) + at * (F32 ? 4 : 2);
    uint32_t u[4];
    if (VEC) return load16(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (F32) {
            u[j] = reinterpret_cast<const volatile uint32_t *>(p)[j];
        } else {
            const volatile unsigned short *h = reinterpret_cast<const volatile unsigned short *>(p) + 2 * j;
            u[j] = (uint32_t)h[0] | (uint32_t)h[1] << 16;
        }
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ uint32_t bf2_round(float a, float b) {  // low half from a
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    return d;
}
template <bool VEC, bool F32>
__device__ __forceinline__ void store_word(void *base, int at, const float *y) {
    char *p = reinterpret_cast<char *>(base) + at * (F32 ? 4 : 2);
    uint32_t u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = F32 ? __float_as_uint(y[j]) : bf2_round(y[2 * j], y[2 * j + 1]);
    if (VEC) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(u[0], u[1], u[2], u[3]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (F32) {
                reinterpret_cast<uint32_t *>(p)[j] = u[j];
            } else {
                unsigned short *h = reinterpret_cast<unsigned short *>(p) + 2 * j;
                h[0] = (unsigned short)u[j], h[1] = (unsigned short)(u[j] >> 16);
            }
        }
    }
}

__device__ __forceinline__ float weight_at(const TurnWeight &w, long long at) {
    if (!w.p) return 1.0f;
    return w.f32 ? __ldg(reinterpret_cast<const float *>(w.p) + at)
                 : __uint_as_float((uint32_t)__ldg(reinterpret_cast<const unsigned short *>(w.p) + at) << 16);
}

// two float32 at once
__device__ __forceinline__ void mul2(float &x, float &y, float a, float b) {
    asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tmul.rn.f32x2 u, u, v;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(x), "+f"(y)
        : "f"(a), "f"(b));
}
__device__ __forceinline__ void fma2(float &x, float &y, float a, float b, float c, float d) {  // x += a c, y += b d
    asm("{\n\t.reg .b64 u, v, w;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tmov.b64 w, {%4, %5};\n\t"
        "fma.rn.f32x2 u, v, w, u;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(x), "+f"(y)
        : "f"(a), "f"(b), "f"(c), "f"(d));
}

// four neighbouring weights (vec: of a row on the 16-byte grid)
__device__ __forceinline__ float4 weight4(const TurnWeight &w, long long at) {
    if (!w.p) return make_float4(1.0f, 1.0f, 1.0f, 1.0f);
    if (w.vec && w.f32) return __ldg(reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(w.p) + at));
    if (w.vec) {
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(reinterpret_cast<const unsigned short *>(w.p) + at));
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                           __uint_as_float(v.y & 0xFFFF0000u));
    }
    return make_float4(weight_at(w, at), weight_at(w, at + 1), weight_at(w, at + 2), weight_at(w, at + 3));
}

// Position of token i of sequence b on an axis.
__device__ __forceinline__ int turn_position(const Turn &a, int b, int i, int axis) {
    if (a.positions) return __ldg(a.positions + ((size_t)axis * a.B + b) * a.n + i);
    // (wraps as unsigned beyond 2^31: no position a caller can mean)
    return (int)((unsigned)(a.start ? __ldg(a.start + b) : 0) + (unsigned)(a.base ? __ldg(a.base + b) : 0) +
                 (unsigned)(a.depth ? __ldg(a.depth + b * a.depth_b + i) : i));
}
__device__ __forceinline__ int turn_axis(const Turn &a, int j) {
    return a.axes && a.positions ? min(max(__ldg(a.axes + j), 0), a.n_axes - 1) : 0;
}

// Where the numbers of lane l of a row's LN lie: y[c][w * PC ..] are the PC channels from
// chan(c, w) on, 16 bytes of a row, w < W.  Half-split pairs have their channels at one
// place of y[0] and y[1].  GROUPS: whole groups.  FULL: all channels turn.
template <int D, bool F32, bool INTER, bool FULL, bool GROUPS>
struct Lane {
    static constexpr int G = D / KV4_GROUPS, PC = F32 ? 4 : 8, LN = GROUPS ? 4 : D / 16, HC = D / (2 * LN), W = HC / PC;
    int l, R;
    __device__ __forceinline__ int chan(int c, int w) const {
        const int half = FULL ? D / 2 : R / 2;
        if (GROUPS) {
            const int h = half / G;
            return (!INTER && (FULL || l < h) ? l + (c ? h : 0) : 2 * l + c) * G + w * PC;
        }
        const int k = (l + LN * w) * PC;
        if (INTER) return k + (c ? D / 2 : 0);
        return FULL || k < half ? k + (c ? half : 0) : k + (c ? D / 2 : half);
    }
    __device__ __forceinline__ bool turns(int c, int w) const { return FULL || chan(c, w) < R; }
};

// ---------------------------------------------------------------------------
// Codes of a group of z whose numbers are within E of the 64-bit ones: false where those
// could have other codes, or float32 had none.
template <int G>
__device__ __forceinline__ bool quantise_near(const float (&z)[G], float E, uint32_t (&w)[G / 8], float *t_out) {
    float mx = z[0], mn = z[0];
#pragma unroll
    for (int i = 1; i < G; i += 2) {
        const float y = z[i], u = z[i + 1 < G ? i + 1 : i];
        asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(mx) : "f"(y), "f"(u));
        asm("min.NaN.f32 %0, %0, %1, %2;" : "+f"(mn) : "f"(y), "f"(u));
    }
    // (products of finite numbers may pass float32, and the numbers beside one that is none
    // have their codes too)
    const bool finite = mx <= FLT_MAX && mn >= -FLT_MAX;
    const float big = fmaxf(mx, -mn);
    const float t = kv4_t(mx > -mn ? fminf(mx, KV4_CAP) : fmaxf(mn, -KV4_CAP)), s = t * KV4_STEP;
    const bool none = big + E < KV4_TINY;  // (a group of zeros among them)
    // (magnitudes beyond what a row holds are alike: the first of them decides)
    const bool sure = fabsf(mx + mn) > 2.0f * E && big + E <= KV4_CAP && kv4_t(big + E) == kv4_t(fmaxf(big - E, 0.0f));
    const float inv = s == 0.0f ? 0.0f : __frcp_rn(s);
    constexpr float BIG = 12582912.0f;
    float far = 0.0f;
#pragma unroll
    for (int i = 0; i < G / 8; ++i) {
        w[i] = KV4_BITS;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = z[8 * i + e];
            const float r = fmaf(x, inv, BIG);
            far = fmaxf(far, fabsf(fmaf(x, inv, BIG - r)));  // how far the quotient is from its whole number
            w[i] += __float_as_uint(fminf(fmaxf(r, BIG - 8.0f), BIG + 7.0f)) << (4 * (e >> 1) + 16 * (e & 1));
        }
    }
    *t_out = t;
    // E in steps, and the quotient's own roundings (8.25 * 2^-24, and those of the test)
    return finite && (none || (sure && far < 0.5f - fmaf(E, fabsf(inv), 1.0e-6f)));
}

// The angle p f of pair j as 64 bits round it
__device__ __forceinline__ double turn_angle(const Turn &a, int p, int j) { return (double)p * (double)__ldg(a.freq + j); }
constexpr float TURN_FAR = 67108864.0f;  // 2^26: beyond it that rounding shows

// 1 / (2 pi) in two parts
constexpr double INV_TURN = 0.15915494309189535, INV_TURN_LO = -9.839338337591493e-18;

// A row again in float64, whatever its numbers and weights are, by a whole warp: a lane has
// D / 32 neighbouring channels, four lanes a group.  True where a number is none.
template <int D, bool F32, bool INTER>
static __device__ __noinline__ bool wide_row(const Turn &a, int b, int i, int h, uint8_t *row) {
    constexpr int G = D / KV4_GROUPS, CH = D / 32;
    constexpr uint32_t ALL = 0xffffffffu;
    const int lane = threadIdx.x & 31, d0 = lane * CH, half = a.R / 2;
    const long long at = b * a.k.b + i * a.k.i + h * a.k.h + d0;
    double y[CH], ss = 0.0;
    bool none = !a.norm;
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        y[e] = F32 ? reinterpret_cast<const float *>(a.k.p)[at + e]
                   : __uint_as_float((uint32_t) reinterpret_cast<const unsigned short *>(a.k.p)[at + e] << 16);
        none = a.norm ? none || !(fabs(y[e]) <= FLT_MAX) : none && y[e] != y[e];
        ss = fma(y[e], y[e], ss);
        if (a.norm) y[e] *= (double)weight_at(a.kw, h * a.kw.h + d0 + e);
    }
    if (a.norm ? __any_sync(ALL, none) : __all_sync(ALL, none)) {  // a norm that is none leaves zeros and NaN
        if (d0 % 8 == 0) reinterpret_cast<uint32_t *>(row)[d0 / 8] = 0x88888888u;
        if (d0 % G == 0) reinterpret_cast<unsigned short *>(row + D / 2)[d0 / G] = 0;
        return true;
    }
    if (a.norm) {
        for (int x = 16; x > 0; x >>= 1) ss += __shfl_xor_sync(ALL, ss, x);
        const double norm = sqrt(ss / D + a.eps);
#pragma unroll
        for (int e = 0; e < CH; ++e) y[e] /= norm;
    }
    const bool turns = d0 < a.R, second = !INTER && d0 >= half;
    const int other = INTER || !turns ? lane : second ? lane - half / CH : lane + half / CH;
    double z[CH];
    bool bad = false;
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        const double yo = INTER ? y[e ^ 1] : __shfl_sync(ALL, y[e], other);
        z[e] = y[e];
        if (turns) {
            const int j = INTER ? (d0 + e) / 2 : second ? d0 - half + e : d0 + e;
            const double angle = turn_angle(a, turn_position(a, b, i, turn_axis(a, j)), j);
            const double hi = angle * INV_TURN, lo = fma(angle, INV_TURN, -hi) + angle * INV_TURN_LO;  // turns, in two parts
            double sn, cn;
            sincospi(2.0 * (hi - rint(hi) + lo), &sn, &cn);
            const bool v = INTER ? e & 1 : second;
            z[e] = a.scale * (v ? y[e] * cn + yo * sn : y[e] * cn - yo * sn);
        }
        bad |= !(fabs(z[e]) <= DBL_MAX);
        z[e] = z[e] == z[e] ? fmin(fmax(z[e], -(double)KV4_CAP), (double)KV4_CAP) : 0.0;
    }
    double top = z[0];  // the group's first of the largest
#pragma unroll
    for (int e = 1; e < CH; ++e)
        if (fabs(z[e]) > fabs(top)) top = z[e];
#pragma unroll
    for (int x = 1; x < 4; x <<= 1) {
        const double o = __shfl_xor_sync(ALL, top, x);
        if (lane & x ? !(fabs(top) > fabs(o)) : fabs(o) > fabs(top)) top = o;
    }
    double t = 0.0;  // kv4_t()
    if (fabs(top) >= (double)KV4_TINY) {
        const unsigned long long u = (unsigned long long)__double_as_longlong(top * -0x1p-19);
        t = __longlong_as_double((long long)((u + ((1ull << 47) - 1) + (u >> 48 & 1)) & ~((1ull << 48) - 1)));
    }
    const double s = t * (double)KV4_STEP;
    uint32_t w = 0u;
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        const int c = (d0 + e) & 7, r = s == 0.0 ? 0 : (int)fmin(fmax(rint(z[e] / s), -8.0), 7.0);
        w |= (uint32_t)(r + 8) << (4 * (c >> 1) + 16 * (c & 1));
    }
#pragma unroll
    for (int x = 1; x < 8 / CH; x <<= 1) w |= __shfl_xor_sync(ALL, w, x);
    if (d0 % 8 == 0) reinterpret_cast<uint32_t *>(row)[d0 / 8] = w;
    if (d0 % G == 0) reinterpret_cast<unsigned short *>(row + D / 2)[d0 / G] = (unsigned short)(__float_as_uint((float)t) >> 16);
    return __any_sync(ALL, bad);
}

// A row again, to some 46 bits, and into the cache, by a whole warp: a lane has D / 32
// neighbouring channels, four lanes a group.  Rows whose products could leave float32, and
// those with a number within 2^-40 of a border, are left to wide_row(): false.
template <int D, bool F32, bool INTER>
static __device__ __noinline__ bool exact_row(const Turn &a, int b, int i, int h, uint8_t *row) {
    constexpr int G = D / KV4_GROUPS, CH = D / 32;
    constexpr uint32_t ALL = 0xffffffffu;
    const int lane = threadIdx.x & 31, d0 = lane * CH, half = a.R / 2;
    const long long at = b * a.k.b + i * a.k.i + h * a.k.h + d0;
    // Within these limits no product passes float32, and none loses its lower half.
    Two y[CH];
    float xs[CH];
    bool far = false;
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        xs[e] = F32 ? reinterpret_cast<const float *>(a.k.p)[at + e]
                    : __uint_as_float((uint32_t) reinterpret_cast<const unsigned short *>(a.k.p)[at + e] << 16);
        y[e] = {xs[e], 0.0f};
        far |= !(fabsf(xs[e]) <= 0x1p55f);
        if (a.norm) {
            const float wt = weight_at(a.kw, h * a.kw.h + d0 + e);
            y[e] = two_product(xs[e], wt);  // (exact: equal ones stay equal)
            far |= !(fabsf(wt) <= 0x1p60f) || (fabsf(y[e].h) < 0x1p-100f && xs[e] != 0.0f && wt != 0.0f);
        }
    }
    if (__any_sync(ALL, far)) return false;
    if (a.norm) {
        Two ss = {0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < CH; ++e) ss = ss + two_product(xs[e], xs[e]);
        for (int x = 16; x > 0; x >>= 1) ss = ss + Two{__shfl_xor_sync(ALL, ss.h, x), __shfl_xor_sync(ALL, ss.l, x)};
        const Two r = two_rsqrt(Two{ss.h / D, ss.l / D} + Two{a.eps32, a.eps_low});
#pragma unroll
        for (int e = 0; e < CH; ++e) y[e] = y[e] * r;
    }
    // A lane works out half of its pairs' cosines and sines: interleaved pairs are its own,
    // the others are shared with the lane that has their other channels.  (The angle is
    // rounded as a product in 64 bits is.)
    const bool turns = d0 < a.R, second = !INTER && d0 >= half;
    const int other = INTER || !turns ? lane : second ? lane - half / CH : lane + half / CH;
    Two sn[CH / 2], cn[CH / 2];
#pragma unroll
    for (int x = 0; x < CH / 2; ++x) {
        sn[x] = {0.0f, 0.0f}, cn[x] = {1.0f, 0.0f};
        if (!turns) continue;
        const int j = INTER ? d0 / 2 + x : second ? d0 - half + CH / 2 + x : d0 + x;
        const double angle = turn_angle(a, turn_position(a, b, i, turn_axis(a, j)), j);
        const double hi = angle * INV_TURN, lo = fma(angle, INV_TURN, -hi) + angle * INV_TURN_LO;  // turns, in two parts
        const double t = hi - rint(hi) + lo;
        const float th = (float)t;
        two_sincos({th, (float)(t - th)}, sn[x], cn[x]);
    }
    Two z[CH];
    auto turned = [&](Two u, Two v, Two c, Two s) { return u * c + -(v * s); };
    if (INTER) {
#pragma unroll
        for (int x = 0; x < CH / 2; ++x) {
            z[2 * x] = turned(y[2 * x], y[2 * x + 1], cn[x], sn[x]);
            z[2 * x + 1] = turned(y[2 * x + 1], -y[2 * x], cn[x], sn[x]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            const int x = e % (CH / 2);
            const bool mine = (e >= CH / 2) == second;
            const Two yo = {__shfl_sync(ALL, y[e].h, other), __shfl_sync(ALL, y[e].l, other)};
            const Two so = {__shfl_sync(ALL, sn[x].h, other), __shfl_sync(ALL, sn[x].l, other)};
            const Two co = {__shfl_sync(ALL, cn[x].h, other), __shfl_sync(ALL, cn[x].l, other)};
            z[e] = turned(y[e], second ? -yo : yo, mine ? cn[x] : co, mine ? sn[x] : so);
        }
    }
    Two top = {0.0f, 0.0f};
    auto larger = [](Two p, Two q) {  // in magnitude
        const float ph = fabsf(p.h), qh = fabsf(q.h);
        return ph > qh || (ph == qh && copysignf(1.0f, p.h) * p.l > copysignf(1.0f, q.h) * q.l);
    };
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        z[e] = !turns ? y[e] : a.scale == 1.0 ? z[e] : z[e] * Two{a.scale32, a.scale_low};
        if (larger(z[e], {KV4_CAP, 0.0f})) z[e] = {copysignf(KV4_CAP, z[e].h), 0.0f};
        if (larger(z[e], top)) top = z[e];  // the first of the largest
    }
#pragma unroll
    for (int x = 1; x < 4; x <<= 1) {
        const Two o = {__shfl_xor_sync(ALL, top.h, x), __shfl_xor_sync(ALL, top.l, x)};
        if (lane & x ? !larger(top, o) : larger(o, top)) top = o;
    }
    // The step: kv4_t() of the first part, but that where this lies on a half the second
    // one decides.
    float t = larger({KV4_TINY, 0.0f}, top) ? 0.0f : kv4_t(top.h);
    // Numbers that are not exact here, and this close to a border, may be rounded onto it or
    // across it in float64 (5 times a scale of 1.2 is 6 there): wide_row() has them.
    const bool exact = !turns || a.scale == 1.0;
    auto close = [&](float off, Two x) { return fabsf(off) < 0x1p-40f * fabsf(x.h) && (a.norm || !exact || x.l != 0.0f); };
    bool unclear = t != 0.0f && (__float_as_uint(top.h) & 0x7FFFFu) == 0x40000u && close(top.l, top);
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        // of the other sign, and as large or nearly: the step's sign is float64's (equal numbers are
        // equal there too, but where a norm or a scale has rounded a turn's share away)
        const float off = (z[e].h + top.h) + (z[e].l + top.l);
        unclear |= t != 0.0f && fabsf(off) < 0x1p-40f * fabsf(top.h) && (off != 0.0f || (turns && (a.norm || a.scale != 1.0)));
    }
    if (t != 0.0f && top.l != 0.0f && (__float_as_uint(top.h) & 0x7FFFFu) == 0x40000u) {
        const bool up = (top.l > 0.0f) == (top.h > 0.0f);
        const uint32_t u = __float_as_uint(top.h * -1.9073486328125e-06f) & ~0x7FFFFu;  // -2^-19
        t = __uint_as_float(u + (up ? 0x80000u : 0u));
    }
    const float s = t * KV4_STEP, inv = s == 0.0f ? 0.0f : __frcp_rn(s), hs = 0.5f * fabsf(s);
    uint32_t w = 0u;
#pragma unroll
    for (int e = 0; e < CH; ++e) {
        const int c = (d0 + e) & 7;  // of its word
        float r = rintf(z[e].h * inv);
        const float d = fmaf(-r, s, z[e].h);  // exact, on the grid of the halves
        const bool along = (z[e].l > 0.0f) == (d > 0.0f);
        unclear |= hs != 0.0f && close(fabsf(d) - hs + (along ? fabsf(z[e].l) : -fabsf(z[e].l)), z[e]);
        if (fabsf(d) > hs || (fabsf(d) == hs && hs != 0.0f && (z[e].l == 0.0f ? ((int)r & 1) : along))) r += (d > 0.0f) == (s > 0.0f) ? 1.0f : -1.0f;
        w |= (uint32_t)((int)fminf(fmaxf(r, -8.0f), 7.0f) + 8) << (4 * (c >> 1) + 16 * (c & 1));
    }
    if (__any_sync(ALL, unclear)) return false;
#pragma unroll
    for (int x = 1; x < 8 / CH; x <<= 1) w |= __shfl_xor_sync(ALL, w, x);
    if (d0 % 8 == 0) reinterpret_cast<uint32_t *>(row)[d0 / 8] = w;
    if (d0 % G == 0) reinterpret_cast<unsigned short *>(row + D / 2)[d0 / G] = (unsigned short)(__float_as_uint(t) >> 16);
    return true;
}

// ---------------------------------------------------------------------------
template <bool VEC, bool F32, class My>
__device__ __forceinline__ void load_row(const My my, const TurnHeads &from, int b, int i, int h, uint4 (&raw)[2][My::W]) {
    const char *p = reinterpret_cast<const char *>(from.p) + (b * from.b + i * from.i + h * from.h) * (F32 ? 4 : 2);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int w = 0; w < My::W; ++w) raw[c][w] = load_word<VEC, F32>(p, my.chan(c, w));
}
template <bool F32, int W, int HC>
__device__ __forceinline__ void numbers(const uint4 (&raw)[2][W], float (&y)[2][HC]) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < HC; ++e) y[c][e] = Elem<F32 ? ACES_F32 : ACES_BF16>::get(raw[c][e / (F32 ? 4 : 8)], e % (F32 ? 4 : 8));
}

// The sum of a row's squares, whose lanes are LN neighbours: eight sums a lane, then a tree.
template <int LN, int HC>
__device__ __forceinline__ float squares(const float (&y)[2][HC]) {
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = y[0][e];
#pragma unroll
    for (int e = 0; e < 8; e += 2) mul2(p[e], p[e + 1], p[e], p[e + 1]);
#pragma unroll
    for (int e = 8; e < 2 * HC; e += 2) {
        const float *v = &y[e / HC][e % HC];
        fma2(p[e % 8], p[e % 8 + 1], v[0], v[1], v[0], v[1]);
    }
    float ss = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
    for (int x = 1; x < LN; x <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, x);
    return ss;
}

// 1 / the norm of a row, whose lanes are LN neighbours.  Numbers whose squares pass
// float32 become 2^-70 of themselves, and are summed in the same order.
template <int D, int LN, int HC>
__device__ __forceinline__ float inv_norm(const Turn &a, float (&y)[2][HC]) {
    float ss = squares<LN>(y);
    const bool huge = !(ss < 1e37f);
    float eps = a.eps32;
    if (__any_sync(0xffffffffu, huge)) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < HC; ++e)
                if (huge) y[c][e] *= 0x1p-70f;
        const float s2 = squares<LN>(y);
        if (huge) ss = s2, eps = 0.0f;
    }
    // (a Newton step behind the approximation: within 1.5 * 2^-24)
    const float m = fmaf(ss, 1.0f / D, eps), r = rsqrtf(m);
    return m <= FLT_MAX ? fmaf(-0.5f * r, fmaf(m * r, r, -1.0f), r) : r;
}

// Turns four numbers of y[c] from e on: half-split pairs with those of y[1] (c = 0), or
// interleaved among themselves; cc and sc: their four or two cosines and sines.
template <bool INTER, int HC>
__device__ __forceinline__ void turn4(float (&y)[2][HC], int c, int e, const float *cc, const float *sc) {
    if (INTER) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float u = y[c][e + 2 * x], v = y[c][e + 2 * x + 1];
            y[c][e + 2 * x] = fmaf(u, cc[x], -(v * sc[x]));
            y[c][e + 2 * x + 1] = fmaf(v, cc[x], u * sc[x]);
        }
    } else {
#pragma unroll
        for (int x = 0; x < 4; x += 2) {
            const float u0 = y[0][e + x], u1 = y[0][e + x + 1], v0 = y[1][e + x], v1 = y[1][e + x + 1];
            float m0 = v0, m1 = v1, n0 = u0, n1 = u1;
            mul2(m0, m1, sc[x], sc[x + 1]);
            mul2(n0, n1, sc[x], sc[x + 1]);
            y[0][e + x] = fmaf(u0, cc[x], -m0), y[0][e + x + 1] = fmaf(u1, cc[x + 1], -m1);
            fma2(n0, n1, v0, v1, cc[x], cc[x + 1]);
            y[1][e + x] = n0, y[1][e + x + 1] = n1;
        }
    }
}

// What a warp works on: tokens [i0, i0 + tokens) of a sequence, and a share of their rows:
// of those for the cache all, in the first slice, which has the tokens' status; of the
// others steps [s0, s1) of every token (keys, then queries; RW heads a step).
struct Unit {
    int b, i0, tokens, slice, s0, s1;
};
struct Units {
    uint32_t per, whole, units, stride;  // of a sequence, of a slice, in all; from one of a warp's to its next
    int T, slices, first, ks, steps;     // first: slices without steps
    __device__ __forceinline__ Unit at(const Turn &a, uint32_t x) const {
        Unit u;
        // (all first slices, which cost the most, before the others)
        const uint32_t share = slices > 1 ? x / whole : 0, unit = x - share * whole;
        u.slice = (int)share, u.b = (int)(unit / per), u.i0 = (int)(unit - u.b * per) * T, u.tokens = min(T, a.n - u.i0);
        u.s0 = 0, u.s1 = steps;
        if (slices > 1) {
            u.s0 = u.slice < first ? 0 : steps * (u.slice - first) / (slices - first);
            u.s1 = u.slice < first ? 0 : steps * (u.slice - first + 1) / (slices - first);
        }
        return u;
    }
};

// The steps of a rotation's warp in their order, DEPTH of them under way into the warp's ring
// in shared memory: each lane copies its own numbers and reads them back, so nothing but
// its own copies is waited for.
template <int D, bool F32, bool INTER, bool FULL>
struct Feed {
    using My = Lane<D, F32, INTER, FULL, false>;
    static constexpr int W = My::W, LN = My::LN, RW = 32 / LN, DEPTH = F32 ? 2 : 4, RING = DEPTH * 2 * W * 512;
    Units all;
    Unit u;
    uint32_t x, ring;
    int s, tok, put, get;
    __device__ __forceinline__ void open(const Turn &a) {
        for (; x < all.units; x += all.stride) {
            u = all.at(a, x);
            if (u.s0 < u.s1) break;
        }
        s = u.s0, tok = 0;
    }
    __device__ __forceinline__ void start(const Turn &a, const Units &w, uint32_t x0, uint32_t place) {
        all = w, x = x0, ring = place + (threadIdx.x & 31) * 16, put = get = 0;
        u = Unit{0, 0, 0, 0, 0, 0};
        open(a);
        for (int p = 0; p < DEPTH; ++p) ask(a);
    }
    __device__ __forceinline__ void ask(const Turn &a) {
        if (x < all.units) {
            const int lane = threadIdx.x & 31;
            const My my{lane % LN, FULL ? D : a.R};
            const bool q = s >= all.ks;
            const TurnHeads &from = q ? a.q : a.k;
            // (lanes without a head have the last one's numbers)
            const int h = min((q ? s - all.ks : s) * RW + lane / LN, (q ? a.Hq : a.H) - 1);
            const char *p = reinterpret_cast<const char *>(from.p) + (u.b * from.b + (u.i0 + tok) * from.i + h * from.h) * (F32 ? 4 : 2);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int w = 0; w < W; ++w)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + (put * 2 * W + c * W + w) * 512),
                                 "l"(p + my.chan(c, w) * (F32 ? 4 : 2))
                                 : "memory");
            if (++s == u.s1) {
                s = u.s0;
                if (++tok == u.tokens) x += all.stride, open(a);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        put = put + 1 == DEPTH ? 0 : put + 1;
    }
    __device__ __forceinline__ void take(uint4 (&r)[2][W]) {
        asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int w = 0; w < W; ++w)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(r[c][w].x), "=r"(r[c][w].y), "=r"(r[c][w].z), "=r"(r[c][w].w)
                             : "r"(ring + (get * 2 * W + c * W + w) * 512)
                             : "memory");
        get = get + 1 == DEPTH ? 0 : get + 1;
    }
};

// Heads of one token that stay numbers, steps [s0, s1).  ws: weights that all heads share;
// cs: the token's cosines and sines.
template <int D, bool F32, bool APPEND, bool INTER, bool VEC, bool FULL>
__device__ __forceinline__ void turn_heads(const Turn &a, Feed<D, F32, INTER, FULL> &feed, const TurnHeads &from, const TurnHeads &to,
                                           const TurnWeight &wt, const float *ws, const float *cs, int b, int i, int heads, int s0, int s1) {
    using My = Lane<D, F32, INTER, FULL, false>;
    constexpr int HC = My::HC, PC = My::PC, LN = My::LN, RW = 32 / LN, W = My::W;
    static_assert(HC == 8, "16 channels a lane");
    const int lane = threadIdx.x & 31;
    const My my{lane % LN, FULL ? D : a.R};
    // (a rotation's steps come through the ring, whose code costs the write more registers than it has)
    constexpr bool RING = VEC && !APPEND;
    constexpr int ES = F32 ? 4 : 2;
    const int row = lane / LN;
    uint4 r[2][W];
    if (!RING) load_row<VEC, F32>(my, from, b, i, min(s0 * RW + row, heads - 1), r);
    char *dst = reinterpret_cast<char *>(to.p) + (b * to.b + i * to.i) * ES;
    // A pair's turn and weights in one: z_u = x_u ta + x_v tb, z_v = x_v tc + x_u td.  Pair
    // e: y[0][e], y[1][e], or interleaved y[e / 4][2 (e % 4)] and its neighbour.  Numbers
    // that do not turn have ta and tc, their weights.
    float ta[HC], tb[HC], tc[HC], td[HC];
    auto tables = [&](int h) {
#pragma unroll
        for (int e = 0; e < HC; e += 4) {
            float wu[4] = {1.0f, 1.0f, 1.0f, 1.0f}, wv[4] = {1.0f, 1.0f, 1.0f, 1.0f}, cc[4] = {1.0f, 1.0f, 1.0f, 1.0f}, sc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            const int c = INTER ? e / 4 : 0, n0 = INTER ? 0 : e;  // numbers y[c][n0 ..]
            const int d = my.chan(c, n0 / PC) + n0 % PC, dv = INTER ? my.chan(c, 4 / PC) + 4 % PC : my.chan(1, n0 / PC) + n0 % PC;
            if (a.norm) {
                const float4 p = wt.h == 0 ? *reinterpret_cast<const float4 *>(ws + d) : weight4(wt, h * wt.h + d);
                const float4 q = wt.h == 0 ? *reinterpret_cast<const float4 *>(ws + dv) : weight4(wt, h * wt.h + dv);
                if (INTER) {
                    wu[0] = p.x, wv[0] = p.y, wu[1] = p.z, wv[1] = p.w, wu[2] = q.x, wv[2] = q.y, wu[3] = q.z, wv[3] = q.w;
                } else {
                    wu[0] = p.x, wu[1] = p.y, wu[2] = p.z, wu[3] = p.w, wv[0] = q.x, wv[1] = q.y, wv[2] = q.z, wv[3] = q.w;
                }
            }
#pragma unroll
            for (int x = 0; x < 4; x += 2) {  // (interleaved pairs of float32 may have one 16 bytes that turn and one that do not)
                const int n = INTER ? 2 * x : e + x, at = my.chan(c, n / PC) + n % PC;
                if (!my.turns(c, n / PC)) continue;
                const float2 cv = *reinterpret_cast<const float2 *>(cs + (INTER ? at / 2 : at));
                const float2 sv = *reinterpret_cast<const float2 *>(cs + D / 2 + (INTER ? at / 2 : at));
                cc[x] = cv.x, cc[x + 1] = cv.y, sc[x] = sv.x, sc[x + 1] = sv.y;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) ta[e + x] = wu[x] * cc[x], tb[e + x] = -(wv[x] * sc[x]), tc[e + x] = wv[x] * cc[x], td[e + x] = wu[x] * sc[x];
        }
    };
    if (!a.norm || wt.h == 0) tables(0);
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        const int h = s * RW + row;
        float y[2][HC];
        if (RING) feed.take(r);
        numbers<F32>(r, y);
        if (RING)
            feed.ask(a);
        else if (s + 1 < s1)
            load_row<VEC, F32>(my, from, b, i, min(h + RW, heads - 1), r);
        float in = 1.0f;
        if (a.norm) {
            in = inv_norm<D, LN>(a, y);
            if (wt.h != 0) tables(min(h, heads - 1));
        }
#pragma unroll
        for (int e = 0; e < HC; e += 2) {
            const int c = INTER ? e / 4 : 0, n = INTER ? 2 * (e % 4) : e;
            float &u0 = y[c][n], &u1 = INTER ? y[c][n + 2] : y[0][n + 1], &v0 = INTER ? y[c][n + 1] : y[1][n], &v1 = INTER ? y[c][n + 3] : y[1][n + 1];
            float p0 = u0, p1 = u1, q0 = v0, q1 = v1;
            mul2(p0, p1, ta[e], ta[e + 1]);
            mul2(q0, q1, tc[e], tc[e + 1]);
            if (my.turns(c, n / PC)) {
                fma2(p0, p1, v0, v1, tb[e], tb[e + 1]);
                fma2(q0, q1, u0, u1, td[e], td[e + 1]);
            }
            if (a.norm) {
                mul2(p0, p1, in, in);
                mul2(q0, q1, in, in);
            }
            u0 = p0, u1 = p1, v0 = q0, v1 = q1;
        }
        if (h >= heads) continue;
        char *p = dst + h * to.h * ES;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int w = 0; w < W; ++w) store_word<VEC, F32>(p, my.chan(c, w), y[c] + w * PC);
    }
}

constexpr int TURN_CTAS = 4;  // an SM, of up to 128 registers a thread

// VEC: every 16 bytes lie on their grid; FULL: all channels turn.
template <int D, bool F32, bool APPEND, bool INTER, bool VEC, bool FULL>
__global__ void __launch_bounds__(TN, TURN_CTAS) k_turn(Turn a, int lt, int slices) {
    constexpr int G = D / KV4_GROUPS, RB = kv4_row_bytes(D), RW = 512 / D;  // RW: heads of a step that stay numbers
    using My = Lane<D, F32, INTER, FULL, true>;
    constexpr int PC = My::PC;
    // weights of queries and keys [D], of each warp [token] cosines, sines [D / 2], and its ring
    extern __shared__ __align__(128) float tables[];
    __shared__ int sts[TW][TOKENS];
    __shared__ uint32_t nears[TW];
    const int T = 1 << lt, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, R = FULL ? D : a.R;
    float *ws = tables, *cs = tables + 2 * D + warp * (T * D);
    int *st = sts[warp];
    const My my{lane & 3, R};

    // The lane's pairs, lane and lane + 32: 2^64 f / (2 pi), whose whole turns do not count
    uint32_t fh[2] = {0u, 0u}, fl[2] = {0u, 0u};
    int axis[2] = {0, 0};
    float fastest = 0.0f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int j = lane + 32 * x;
        if (j >= R / 2) continue;
        fastest = fmaxf(fastest, fabsf(__ldg(a.freq + j)));
        const double f = __ldg(a.freq + j), hi = f * INV_TURN, lo = fma(f, INV_TURN, -hi) + f * INV_TURN_LO;
        const unsigned long long u = __double2ull_rz((hi - floor(hi)) * 0x1p64) + (unsigned long long)__double2ll_rn(lo * 0x1p64);
        fh[x] = (uint32_t)(u >> 32), fl[x] = (uint32_t)u;
        axis[x] = turn_axis(a, j);
    }
    // positions beyond which the angle's rounding to 64 bits shows, of the warp's fastest pair
    fastest = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fastest)));
    if (lane == 0) nears[warp] = fastest > TURN_FAR * 0x1p-31f ? (uint32_t)(TURN_FAR / fastest) : 0x80000000u;
    if (a.norm)  // weights that all heads share
        for (int y = 4 * threadIdx.x; y < 2 * D; y += 4 * TN) {
            const TurnWeight &w = y < D ? a.qw : a.kw;
            if (w.h == 0) *reinterpret_cast<float4 *>(ws + y) = weight4(w, y % D);
        }
    __syncthreads();

    Units all;
    all.per = (uint32_t)(a.n + T - 1) >> lt, all.whole = (uint32_t)a.B * all.per, all.units = all.whole * slices, all.stride = gridDim.x * TW;
    all.T = T, all.slices = slices, all.first = APPEND && slices > 1 ? 1 : 0;
    all.ks = APPEND ? 0 : (a.H + RW - 1) / RW, all.steps = all.ks + (a.Hq + RW - 1) / RW;
    const int ks = all.ks;
    const uint32_t x0 = blockIdx.x * TW + warp;
    using Heads = Feed<D, F32, INTER, FULL>;
    Heads feed;
    if (VEC && !APPEND) feed.start(a, all, x0, (uint32_t)__cvta_generic_to_shared(tables + 2 * D + TW * T * D) + warp * Heads::RING);
    // positions of the lane's pairs, asked for a unit ahead
    int p_next[2];
    auto ask = [&](uint32_t x) {
        if (x >= all.units) return;
        const uint32_t unit = x % all.whole, b = unit / all.per;
#pragma unroll
        for (int y = 0; y < 2; ++y)
            if (lane + 32 * y < R / 2) p_next[y] = turn_position(a, (int)b, (int)(unit - b * all.per) * T, axis[y]);
    };
    ask(x0);
#pragma unroll 1
    for (uint32_t x = x0; x < all.units; x += all.stride) {
        const Unit u = all.at(a, x);
        const int b = u.b, i0 = u.i0, tokens = u.tokens, slice = u.slice, s0 = u.s0, s1 = u.s1;
        const int ok = (tokens * a.H + 7) >> 3;  // eight rows for the cache at a time, keys, then values
        const int octets = APPEND && slice == 0 ? 2 * ok : 0;

        // The row of this lane in an octet: token, head.  Lanes without one (false) have the
        // last one's numbers, and write nothing.
        auto place = [&](int o, int &tok, int &h) {
            const int r = (o < ok ? o : o - ok) * 8 + (lane >> 2), rr = min(r, tokens * a.H - 1);
            tok = tokens == 1 ? 0 : rr / a.H;
            h = rr - tok * a.H;
            return r == rr;
        };
        uint4 raw[2][My::W];
        auto fetch = [&](int o) {
            int tok, h;
            if (o >= octets) return;
            place(o, tok, h);
            load_row<VEC, F32>(my, o < ok ? a.k : a.v, b, i0 + tok, h, raw);
        };
        if (APPEND) fetch(0);

        auto put_turn = [&](int tok, int j, uint32_t turns) {
            float sn, cn;
            // (to 24 bits, 2 pi 2^-26 of the angle: counted below)
            sincospif((float)(int)turns * 0x1p-31f, &sn, &cn);
            cs[tok * D + j] = cn * a.scale32, cs[tok * D + D / 2 + j] = sn * a.scale32;
        };
        uint32_t farthest = 0u;
        __syncwarp();  // the last unit's tables are read
#pragma unroll 1
        for (int tok = 0; tok < tokens; ++tok)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int j = lane + 32 * y;
                if (j >= R / 2) continue;
                const uint32_t p = (uint32_t)(tok == 0 ? p_next[y] : turn_position(a, b, i0 + tok, axis[y]));
                farthest = max(farthest, p >> 31 ? 0u - p : p);
                put_turn(tok, j, p * fh[y] + __umulhi(p, fl[y]) - (p >> 31 ? fl[y] : 0u));
            }
        if (farthest > nears[warp])  // those angles again, with their roundings
#pragma unroll 1
            for (int z = 0; z < 2 * tokens; ++z) {
                const int tok = z >> 1, y = z & 1, j = lane + 32 * y;
                if (j >= R / 2) continue;
                const uint32_t p = (uint32_t)turn_position(a, b, i0 + tok, turn_axis(a, j));
                const double at = (int)p, f = __ldg(a.freq + j);
                put_turn(tok, j, p * (y ? fh[1] : fh[0]) + __umulhi(p, y ? fl[1] : fl[0]) - (p >> 31 ? (y ? fl[1] : fl[0]) : 0u) +
                                     (uint32_t)__double2int_rn(fma(-at, f, at * f) * (INV_TURN * 0x1p32)));
            }
        ask(x + all.stride);
        if (APPEND && lane < TOKENS) st[lane] = 0;
        __syncwarp();

        // (keys, then queries; of a token after another)
#pragma unroll 1
        for (int y = APPEND ? 1 : 0; y < 2 * tokens; y += APPEND ? 2 : 1) {
            const int q = y & 1, tok = y >> 1, from = q ? max(s0 - ks, 0) : s0, to = q ? s1 - ks : min(s1, ks);
            if (from < to)
                turn_heads<D, F32, APPEND, INTER, VEC, FULL>(a, feed, q ? a.q : a.k, q ? a.oq : a.ok, q ? a.qw : a.kw, ws + (q ? 0 : D), cs + tok * D, b, i0 + tok,
                                                     q ? a.Hq : a.H, from, to);
        }
        if (!APPEND) continue;

        const int start = a.start[b], cnt = a.count ? a.count[b] : a.n;
#pragma unroll 1
        for (int o = 0; o < octets; ++o) {
            int tok, h;
            const bool live = place(o, tok, h), keys = o < ok;
            const int i = i0 + tok;
            float y[2][G];
            numbers<F32>(raw, y);
            fetch(o + 1);
            bool bad = false, bad1 = false, sure = true;
            uint32_t w[2][G / 8];
            float t[2];
            const long long pos = (long long)start + i;
            const bool mine = live && i < cnt, in = mine && pos >= 0 && pos < a.S;
            // (numbers that neither turn nor are normed are their own 64-bit ones: bfloat16 ones lie on
            // borders too often to be done again, 264 us for 8192 tokens of 32 and 8 heads, half turned, so 87)
            if (!keys || (!FULL && !a.norm && !my.turns(0, 0))) {
                quantise<G, F32>(y[0], w[0], &t[0], &bad);
                quantise<G, F32>(y[1], w[1], &t[1], &bad1);
            } else {
                if (a.norm) {
                    const float r = inv_norm<D, 4>(a, y);
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < G; e += 4) {
                            const int d = my.chan(c, e / PC) + e % PC;
                            float4 v = a.kw.h == 0 ? *reinterpret_cast<const float4 *>(ws + D + d) : weight4(a.kw, h * a.kw.h + d);
                            mul2(v.x, v.y, r, r);
                            mul2(v.z, v.w, r, r);
                            mul2(y[c][e], y[c][e + 1], v.x, v.y);
                            mul2(y[c][e + 2], y[c][e + 3], v.z, v.w);
                        }
                }
                // Float32's z is within 17 u = 17 * 2^-24 of the 64-bit one, relative to the length h
            // of its pair: the sum of squares 9 u (four in a row, three and two levels more), half
            // of which shows in the root, the mean with eps 0.5 u, the root 1.5 u, r w and its
            // product with x 1 u each: 8.5 u; a product of the two and their sum 2 u; cosine and
            // sine 1 u and 2 pi 2^-26 < 1.6 u of their angle, absolute, for both together 2^0.5
            // as much of h: 3.7 u; the scale's two roundings 2 u.
            // (E: the largest square of a group, or of what turns of pairs among both)
                float E[2] = {0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < G; e += 2) {
                        if (INTER || !my.turns(c, e / PC))
                            E[c] = fmaxf(E[c], fmaf(y[c][e], y[c][e], y[c][e + 1] * y[c][e + 1]));
                        else if (c == 0)
                            E[0] = fmaxf(E[0], fmaxf(fmaf(y[0][e], y[0][e], y[1][e] * y[1][e]), fmaf(y[0][e + 1], y[0][e + 1], y[1][e + 1] * y[1][e + 1])));
                    }
                if (!INTER && my.turns(0, 0)) E[1] = E[0];
#pragma unroll
                for (int c = 0; c < (INTER ? 2 : 1); ++c)
#pragma unroll
                    for (int e = 0; e < G; e += 4) {
                        if (!my.turns(c, e / PC)) continue;
                        const float *cp = cs + tok * D + (my.chan(c, e / PC) + e % PC) / (INTER ? 2 : 1);
                        float cc[4], sc[4];
                        if (INTER) {
                            const float2 cv = *reinterpret_cast<const float2 *>(cp), sv = *reinterpret_cast<const float2 *>(cp + D / 2);
                            cc[0] = cv.x, cc[1] = cv.y, sc[0] = sv.x, sc[1] = sv.y;
                        } else {
                            const float4 cv = *reinterpret_cast<const float4 *>(cp), sv = *reinterpret_cast<const float4 *>(cp + D / 2);
                            cc[0] = cv.x, cc[1] = cv.y, cc[2] = cv.z, cc[3] = cv.w, sc[0] = sv.x, sc[1] = sv.y, sc[2] = sv.z, sc[3] = sv.w;
                        }
                        turn4<INTER>(y, c, e, cc, sc);
                    }
                float near[2];
#pragma unroll
                for (int c = 0; c < 2; ++c)  // (the least length: of squares below float32)
                    near[c] = fmaxf(__fsqrt_rn(E[c]), 1e-22f) * (my.turns(c, 0) ? a.scale32 : 1.0f) * 0x1.1p-20f;
                sure = quantise_near<G>(y[0], near[0], w[0], &t[0]);
                sure &= quantise_near<G>(y[1], near[1], w[1], &t[1]);
            }
            if (mine && !in) atomicOr(&st[tok], ACES_ROW_RANGE);
            if (in && (bad || bad1)) atomicOr(&st[tok], ACES_ROW_NONFINITE);
            // rows to be done again: one bit for each of the eight
            uint32_t again = __ballot_sync(0xffffffffu, in && !sure);
            again = (again | again >> 1 | again >> 2 | again >> 3) & 0x11111111u;
            uint8_t *row = nullptr;
            if (in && ACES_IN(pos, a.S)) {
                row = (keys ? a.ck : a.cv) + ((size_t)((size_t)b * a.H + h) * a.S + (size_t)pos) * RB;
                if (!(again >> (lane & ~3) & 1u)) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int g = my.chan(c, 0) / G;
                        uint32_t *to = reinterpret_cast<uint32_t *>(row) + g * (G / 8);
                        if (G == 16)
                            *reinterpret_cast<uint2 *>(to) = make_uint2(w[c][0], w[c][G / 8 - 1]);
                        else
                            *to = w[c][0];
                        reinterpret_cast<unsigned short *>(row + D / 2)[g] = (unsigned short)(__float_as_uint(t[c]) >> 16);
                    }
                }
            }
            for (; again; again &= again - 1) {
                const int from = __ffs(again) - 1;
                uint8_t *to = reinterpret_cast<uint8_t *>(__shfl_sync(0xffffffffu, (unsigned long long)row, from));
                const int ri = __shfl_sync(0xffffffffu, i, from), rh = __shfl_sync(0xffffffffu, h, from);
                if (to && !exact_row<D, F32, INTER>(a, b, ri, rh, to) && wide_row<D, F32, INTER>(a, b, ri, rh, to) && lane == 0)
                    atomicOr(&st[ri - i0], ACES_ROW_NONFINITE);
            }
        }
        if (slice == 0) {
            __syncwarp();
            if (lane < tokens) a.status[(size_t)b * a.n + i0 + lane] = st[lane];
        }
    }
}

// Tokens of a warp (their logarithm): with few key heads several, so that the eight rows
// that go to the cache at a time are not mostly none, while there are warps enough.
static int turn_tokens(const Turn &a, bool append, int nsm) {
    int lt = 0;
    while (append && (2 << lt) <= TOKENS && (a.H << lt) < 8 && (long long)a.B * a.n >= (16ll * nsm) << lt) ++lt;
    return lt;
}

template <int D, bool F32, bool APPEND, bool INTER>
static cudaError_t run_turn(const Turn &a, int nsm, cudaStream_t s) {
    const int lt = turn_tokens(a, APPEND, nsm);
    const long long units = (long long)a.B * ((a.n + (1 << lt) - 1) >> lt);
    constexpr int RW = 512 / D;
    const int most = APPEND ? 1 + (a.Hq + RW - 1) / RW : (a.H + RW - 1) / RW + (a.Hq + RW - 1) / RW;
    int slices = 1;  // (steps times slices is a 32-bit number in the kernel)
    while (slices < most && units * slices < SLICE_WARPS * nsm && (long long)most * (slices + 1) <= INT_MAX) ++slices;
    const long long want = (units * slices + TW - 1) / TW;
    const unsigned grid = (unsigned)(want < (long long)TURN_CTAS * nsm ? want : (long long)TURN_CTAS * nsm);
    const size_t tables = (size_t)((TW << lt) + 2) * (D * 4) + (a.vec && !APPEND ? TW * Feed<D, F32, INTER, true>::RING : 0);
    const auto fn = !a.vec ? k_turn<D, F32, APPEND, INTER, false, false>
                  : a.R == D ? k_turn<D, F32, APPEND, INTER, true, true>
                             : k_turn<D, F32, APPEND, INTER, true, false>;
    fn<<<grid, TN, tables, s>>>(a, lt, slices);
    return cudaGetLastError();
}

template <int D, bool F32>
static cudaError_t run_kind(const Turn &a, bool append, bool interleaved, int nsm, cudaStream_t s) {
    if (append) return interleaved ? run_turn<D, F32, true, true>(a, nsm, s) : run_turn<D, F32, true, false>(a, nsm, s);
    return interleaved ? run_turn<D, F32, false, true>(a, nsm, s) : run_turn<D, F32, false, false>(a, nsm, s);
}
cudaError_t launch_turn(const Turn &a, int D, bool f32, bool append, bool interleaved, int nsm, cudaStream_t s) {
    if (D == 64) return f32 ? run_kind<64, true>(a, append, interleaved, nsm, s) : run_kind<64, false>(a, append, interleaved, nsm, s);
    return f32 ? run_kind<128, true>(a, append, interleaved, nsm, s) : run_kind<128, false>(a, append, interleaved, nsm, s);
}

#ifdef ACES_CHECKED
cudaError_t check_take_turn(unsigned long long out[3]) { return check_take(out); }
#endif

}  // namespace aces
