// Rotation of queries and keys by their positions, with their norms, and the write of
// the keys so made and of the values into a 4-bit cache (the format: kv4.cuh).
//
//   y = x w / sqrt(mean(x^2) + eps)           (a head's D numbers; without norms y = x)
//   z_u = y_u c_j - y_v s_j, z_v = y_v c_j + y_u s_j     c_j, s_j = scale (cos, sin)(p f_j)
//
// for the pairs j < R / 2 of channels (u, v) = (j, j + R / 2), or (2 j, 2 j + 1); p is the
// position on the pair's axis.  Four lanes have a head's row, two of its eight groups
// each, both channels of every pair among them: no number changes lanes, and a lane that
// writes the cache has whole groups to quantise.  A CTA has some tokens of a sequence with
// all their heads; their cosines and sines are made once and lie in shared memory.
//
// The angle p f is taken in 64 bits (a position of 2^20 has no fraction left in 32), as
// turns: its whole turns go before it is rounded to float32.
//
// The cache's codes are those of z in 64 bits, so that they do not depend on how sums and
// products were ordered here.  Float32's z is within E of that; where a quotient lies
// closer than that to a border, or the step could be another, the row's lanes do the row
// again in 64 bits (four rows of a thousand).
#define ACES_FILE 10  // site numbers of the checked build
#include "kv4_quant.cuh"
#include "turn.cuh"

namespace aces {

constexpr int TN = 256, TW = TN / 32;
constexpr int TOKENS = 8;  // of a CTA, at most

// ---------------------------------------------------------------------------
// loads and stores of one group
template <int G, bool F32>
struct Raw {
    static constexpr int N = G * (F32 ? 4 : 2) / 16;
    uint4 w[N];
};
// (in place, a row is read by the lanes that write it, before they do: a plain load)
__device__ __forceinline__ uint4 load16(const void *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <int G, bool F32>
__device__ __forceinline__ void load_raw(const void *base, long long at, bool vec, Raw<G, F32> &r) {
    constexpr int ES = F32 ? 4 : 2;
    const char *p = reinterpret_cast<const char *>(base) + at * ES;
    if (vec) {
#pragma unroll
        for (int i = 0; i < Raw<G, F32>::N; ++i) r.w[i] = load16(p + 16 * i);
    } else {
#pragma unroll
        for (int i = 0; i < Raw<G, F32>::N; ++i) {
            uint32_t u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (F32) {
                    u[j] = reinterpret_cast<const volatile uint32_t *>(p)[4 * i + j];
                } else {
                    const volatile unsigned short *h = reinterpret_cast<const volatile unsigned short *>(p) + 8 * i + 2 * j;
                    u[j] = (uint32_t)h[0] | (uint32_t)h[1] << 16;
                }
            }
            r.w[i] = make_uint4(u[0], u[1], u[2], u[3]);
        }
    }
}
template <int G, bool F32>
__device__ __forceinline__ float raw_get(const Raw<G, F32> &r, int e) {
    return F32 ? Elem<ACES_F32>::get(r.w[e / 4], e % 4) : Elem<ACES_BF16>::get(r.w[F32 ? 0 : e / 8], e % 8);
}
__device__ __forceinline__ uint32_t bf2_round(float a, float b) {  // low half from a
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    return d;
}
template <int G, bool F32>
__device__ __forceinline__ void store_group(void *base, long long at, bool vec, const float (&y)[G]) {
    constexpr int ES = F32 ? 4 : 2;
    char *p = reinterpret_cast<char *>(base) + at * ES;
#pragma unroll
    for (int i = 0; i < Raw<G, F32>::N; ++i) {
        uint32_t u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = F32 ? __float_as_uint(y[F32 ? 4 * i + j : 0]) : bf2_round(y[F32 ? 0 : 8 * i + 2 * j], y[F32 ? 0 : 8 * i + 2 * j + 1]);
        if (vec) {
            reinterpret_cast<uint4 *>(p)[i] = make_uint4(u[0], u[1], u[2], u[3]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (F32) {
                    reinterpret_cast<uint32_t *>(p)[4 * i + j] = u[j];
                } else {
                    unsigned short *h = reinterpret_cast<unsigned short *>(p) + 8 * i + 2 * j;
                    h[0] = (unsigned short)u[j], h[1] = (unsigned short)(u[j] >> 16);
                }
            }
        }
    }
}

__device__ __forceinline__ float weight_at(const TurnWeight &w, long long at) {
    if (!w.p) return 1.0f;
    return w.f32 ? __ldg(reinterpret_cast<const float *>(w.p) + at)
                 : __uint_as_float((uint32_t)__ldg(reinterpret_cast<const unsigned short *>(w.p) + at) << 16);
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

// The two groups of lane l of a row's four, and whether they turn.  Half-split pairs: one
// group of the first half of the turned channels and its partner of the second; then
// neighbours.
template <int D, bool INTER>
__device__ __forceinline__ void lane_groups(int R, int l, int &c0, int &c1) {
    constexpr int G = D / KV4_GROUPS;
    const int half = R / (2 * G);
    c0 = !INTER && l < half ? l : 2 * l;
    c1 = !INTER && l < half ? l + half : 2 * l + 1;
}

// ---------------------------------------------------------------------------
// Codes of a group of z whose numbers are within E of the 64-bit ones: false where those
// could have other codes.
template <int G>
__device__ __forceinline__ bool quantise_near(float (&z)[G], float E, uint32_t (&w)[G / 8], float *t_out, bool *bad) {
    float mx = z[0], mn = z[0];
#pragma unroll
    for (int i = 1; i < G; i += 2) {
        const float y = z[i], u = z[i + 1 < G ? i + 1 : i];
        asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(mx) : "f"(y), "f"(u));
        asm("min.NaN.f32 %0, %0, %1, %2;" : "+f"(mn) : "f"(y), "f"(u));
    }
    *bad = false;
    if (!(mx <= FLT_MAX && mn >= -FLT_MAX)) {  // not finite: what it is does not hang on roundings
        quantise<G, true>(z, w, t_out, bad);
        return true;
    }
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
    return none || (sure && far < 0.5f - fmaf(E, fabsf(inv), 1.0e-6f));
}

// One number of a row in 64 bits.
template <int D, bool F32, bool INTER>
struct Exact {
    const Turn &a;
    const void *x;
    long long at;   // of the row
    TurnWeight wt;  // and of its weights
    long long wat;
    int b, i;
    double r;       // 1 / the norm
    __device__ __forceinline__ double in(int d) const {
        const long long j = at + d;
        return F32 ? reinterpret_cast<const float *>(x)[j]
                   : __uint_as_float((uint32_t) reinterpret_cast<const unsigned short *>(x)[j] << 16);
    }
    __device__ __forceinline__ double y(int d) const { return a.norm ? in(d) * weight_at(wt, wat + d) * r : in(d); }  // (x w is exact: equal ones stay equal)
    __device__ __forceinline__ double z(int d) const {
        if (d >= a.R) return y(d);
        const int half = a.R / 2, j = INTER ? d >> 1 : d % half;
        const bool second = INTER ? d & 1 : d >= half;
        const double u = y(INTER ? 2 * j : j), v = y(INTER ? 2 * j + 1 : j + half);
        double sn, cs;
        sincos((double)turn_position(a, b, i, turn_axis(a, j)) * (double)__ldg(a.freq + j), &sn, &cs);
        return (second ? v * cs + u * sn : u * cs - v * sn) * a.scale;
    }
};

// Codes of a row's groups g[0], g[1] whose float32 numbers z (within E of the 64-bit ones)
// leave them open: the numbers that may be a group's first of largest magnitude, and those
// next to a border, are worked out in 64 bits.  By the row's four lanes, which share its
// sum of squares.
template <int D, bool F32, bool INTER>
static __device__ __noinline__ void exact_groups(Exact<D, F32, INTER> row, uint32_t mask, const int *g, const float *z, const float *E,
                                                 uint32_t *w, float *t_out) {
    constexpr int G = D / KV4_GROUPS;
    if (row.a.norm) {
        double ss = 0.0;
        for (int c = 0; c < 2; ++c)
            for (int e = 0; e < G; ++e) {
                const double f = row.in(g[c] * G + e);
                ss = fma(f, f, ss);
            }
        ss += __shfl_xor_sync(mask, ss, 1);
        ss += __shfl_xor_sync(mask, ss, 2);
        row.r = 1.0 / sqrt(ss / D + row.a.eps);
    }
    constexpr double CAP = (double)KV4_CAP;
    for (int c = 0; c < 2; ++c) {
        const float *zc = z + c * G;
        float big = 0.0f;
        bool fine = true;
        for (int e = 0; e < G; ++e) {
            big = fmaxf(big, fabsf(zc[e]));
            fine &= fabsf(zc[e]) <= FLT_MAX;
        }
        if (!fine) continue;  // what is not finite is not open
        double top = 0.0;
        for (int e = 0; e < G; ++e)
            if (fabsf(zc[e]) >= fminf(big, KV4_CAP) - 2.0f * E[c]) {
                const double v = fmin(fmax(row.z(g[c] * G + e), -CAP), CAP);
                if (fabs(v) > fabs(top)) top = v;
            }
        // -top / 2^19 in five significant bits, ties to even
        double t = 0.0;
        if (fabs(top) >= (double)KV4_TINY) {
            const unsigned long long bits = (unsigned long long)__double_as_longlong(-top * 1.9073486328125e-06);
            unsigned long long m = bits & 0x7FFFFFFFFFFFFFFFull;
            m = (m + 0x7FFFFFFFFFFFull + ((m >> 48) & 1ull)) & ~0xFFFFFFFFFFFFull;
            t = __longlong_as_double((long long)((bits & 0x8000000000000000ull) | m));
        }
        t_out[c] = (float)t;
        const float s = (float)t * KV4_STEP, inv = s == 0.0f ? 0.0f : __frcp_rn(s);
        for (int j = 0; j < G / 8; ++j) {
            uint32_t word = 0u;
            for (int e = 0; e < 8; ++e) {
                const float x = fminf(fmaxf(zc[8 * j + e], -KV4_CAP), KV4_CAP), q = x * inv;
                float r = rintf(q);
                if (s != 0.0f && fabsf(q - r) >= 0.5f - fmaf(E[c], fabsf(inv), 1.5e-6f))
                    r = (float)rint(fmin(fmax(row.z(g[c] * G + 8 * j + e), -CAP), CAP) / (double)s);
                word |= (uint32_t)((int)fminf(fmaxf(r, -8.0f), 7.0f) + 8) << (4 * (e >> 1) + 16 * (e & 1));
            }
            w[c * (G / 8) + j] = word;
        }
    }
}

// ---------------------------------------------------------------------------
template <int D, bool F32, bool APPEND, bool INTER>
__global__ void __launch_bounds__(TN) k_turn(Turn a, int lt) {
    constexpr int G = D / KV4_GROUPS, RB = kv4_row_bytes(D), P = G + 4;  // a group's place in shared memory: no two lanes on a bank
    __shared__ __align__(16) float cs[TOKENS][2][4 * P], wts[2][KV4_GROUPS * P];
    __shared__ int st[TOKENS];
    const int T = 1 << lt, per = (a.n + T - 1) >> lt;  // CTAs of a sequence
    const int b = blockIdx.x / per, i0 = (blockIdx.x - b * per) * T, tokens = min(T, a.n - i0);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, l = lane & 3;
    const uint32_t mask = 0xFu << (lane & ~3);
    // eight rows of one kind a warp: queries, then keys, then values
    const int oq = (tokens * a.Hq + 7) >> 3, ok = (tokens * a.H + 7) >> 3, octets = oq + (APPEND ? 2 : 1) * ok;
    int c0, c1;
    lane_groups<D, INTER>(a.R, l, c0, c1);

    // the row of this lane in an octet: kind, token, head; false for none
    auto place = [&](int o, int &kind, int &tok, int &h) {
        kind = o < oq ? 0 : o < oq + ok ? 1 : 2;
        const int r = (o - (kind == 0 ? 0 : kind == 1 ? oq : oq + ok)) * 8 + (lane >> 2), heads = kind == 0 ? a.Hq : a.H;
        tok = r / heads;
        h = r - tok * heads;
        return tok < tokens;
    };
    Raw<G, F32> raw[2];
    auto fetch = [&](int o) {
        int kind, tok, h;
        if (o >= octets || !place(o, kind, tok, h)) return;
        const TurnHeads &x = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
        const long long at = b * x.b + (i0 + tok) * x.i + h * x.h;
        load_raw<G, F32>(x.p, at + c0 * G, a.vec, raw[0]);
        load_raw<G, F32>(x.p, at + c1 * G, a.vec, raw[1]);
    };
    fetch(warp);

    for (int x = tid; x < tokens * (a.R / 2); x += TN) {
        const int tok = x / (a.R / 2), j = x - tok * (a.R / 2);
        const double p = turn_position(a, b, i0 + tok, turn_axis(a, j));
        const double angle = p * (double)__ldg(a.freq + j);
        // turns: 1 / (2 pi) in two parts
        const double hi = angle * 0.15915494309189535, lo = fma(angle, 0.15915494309189535, -hi) + angle * -9.839338337591493e-18;
        float sn, cn;
        sincospif(2.0f * (float)(hi - rint(hi) + lo), &sn, &cn);
        const int at = j / G * P + j % G;
        cs[tok][0][at] = cn * (float)a.scale, cs[tok][1][at] = sn * (float)a.scale;
    }
    if (a.norm)
        for (int x = tid; x < 2 * D; x += TN) {
            const int which = x / D, d = x - which * D;
            const TurnWeight &w = which ? a.kw : a.qw;
            if (w.h == 0) wts[which][d / G * P + d % G] = weight_at(w, d);
        }
    if (APPEND && tid < T) st[tid] = 0;
    __syncthreads();
    const int start = APPEND ? a.start[b] : 0, cnt = APPEND && a.count ? a.count[b] : a.n;

    for (int o = warp; o < octets; o += TW) {
        int kind, tok, h;
        const bool live = place(o, kind, tok, h);
        const int i = i0 + tok;
        float y[2][G];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < G; ++e) y[c][e] = live ? raw_get<G, F32>(raw[c], e) : 0.0f;
        fetch(o + TW);
        bool bad = false;
        uint32_t w[2][G / 8];
        float t[2];
        const long long pos = APPEND ? (long long)start + i : 0;
        const bool in = APPEND && live && i < cnt && pos >= 0 && pos < a.S;
        if (APPEND && kind == 2) {
            if (!in) {
                if (live && i < cnt && h == 0 && l == 0) atomicOr(&st[tok], ACES_ROW_RANGE);
                continue;
            }
            bool bad1;
            quantise<G, F32>(y[0], w[0], &t[0], &bad);
            quantise<G, F32>(y[1], w[1], &t[1], &bad1);
            bad |= bad1;
        } else {
            const int tk = live ? tok : 0;
            if (a.norm) {
                float p[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = y[0][e] * y[0][e];
#pragma unroll
                for (int e = 8; e < 2 * G; ++e) p[e % 8] = fmaf(y[e / G][e % G], y[e / G][e % G], p[e % 8]);
                float ss = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
                ss += __shfl_xor_sync(0xffffffffu, ss, 1);
                ss += __shfl_xor_sync(0xffffffffu, ss, 2);
                const bool huge = !(ss < 1e37f);
                float eps = (float)a.eps;
                if (__any_sync(0xffffffffu, huge)) {  // squares beyond float32: of numbers times 2^-70
                    float s2 = 0.0f;
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < G; ++e) {
                            if (huge) y[c][e] *= 0x1p-70f;
                            s2 = fmaf(y[c][e], y[c][e], s2);
                        }
                    s2 += __shfl_xor_sync(0xffffffffu, s2, 1);
                    s2 += __shfl_xor_sync(0xffffffffu, s2, 2);
                    if (huge) ss = s2, eps = 0.0f;
                }
                const float r = __frsqrt_rn(fmaf(ss, 1.0f / D, eps));
                const TurnWeight &wt = kind ? a.kw : a.qw;
                const float *ws = wts[kind];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int g = c ? c1 : c0;
#pragma unroll
                    for (int e = 0; e < G; e += 4) {
                        float4 v;
                        if (wt.h == 0) {
                            v = *reinterpret_cast<const float4 *>(ws + g * P + e);
                        } else {
                            const long long at = (live ? h : 0) * wt.h + g * G + e;
                            v = make_float4(weight_at(wt, at), weight_at(wt, at + 1), weight_at(wt, at + 2), weight_at(wt, at + 3));
                        }
                        y[c][e] *= r * v.x, y[c][e + 1] *= r * v.y, y[c][e + 2] *= r * v.z, y[c][e + 3] *= r * v.w;
                    }
                }
            }
            float E[2] = {0.0f, 0.0f};  // the largest square (of a pair that turns: of both its numbers)
            auto largest = [&](float &m, float u, float v) { m = fmaxf(m, fmaf(u, u, v * v)); };
            const bool keys = APPEND && kind == 1;
            if (!INTER) {
                if (c0 < a.R / (2 * G)) {
                    const float *cp = cs[tk][0] + c0 * P, *sp = cs[tk][1] + c0 * P;
#pragma unroll
                    for (int e = 0; e < G; e += 4) {
                        const float4 cv = *reinterpret_cast<const float4 *>(cp + e), sv = *reinterpret_cast<const float4 *>(sp + e);
                        const float cc[4] = {cv.x, cv.y, cv.z, cv.w}, sc[4] = {sv.x, sv.y, sv.z, sv.w};
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const float u = y[0][e + x], v = y[1][e + x];
                            if (keys) largest(E[0], u, v);
                            y[0][e + x] = fmaf(u, cc[x], -(v * sc[x]));
                            y[1][e + x] = fmaf(v, cc[x], u * sc[x]);
                        }
                    }
                    E[1] = E[0];
                }
            } else {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int g = c ? c1 : c0;
                    if (g * G >= a.R) continue;
                    const int j0 = g * (G / 2);
                    const float *cp = cs[tk][0] + j0 / G * P + j0 % G, *sp = cs[tk][1] + j0 / G * P + j0 % G;
#pragma unroll
                    for (int e = 0; e < G; e += 8) {
                        const float4 cv = *reinterpret_cast<const float4 *>(cp + e / 2), sv = *reinterpret_cast<const float4 *>(sp + e / 2);
                        const float cc[4] = {cv.x, cv.y, cv.z, cv.w}, sc[4] = {sv.x, sv.y, sv.z, sv.w};
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const float u = y[c][e + 2 * x], v = y[c][e + 2 * x + 1];
                            if (keys) largest(E[c], u, v);
                            y[c][e + 2 * x] = fmaf(u, cc[x], -(v * sc[x]));
                            y[c][e + 2 * x + 1] = fmaf(v, cc[x], u * sc[x]);
                        }
                    }
                }
            }
            if (!APPEND || kind == 0) {
                if (live) {
                    const TurnHeads &x = kind == 0 ? a.oq : a.ok;
                    const long long at = b * x.b + i * x.i + h * x.h;
                    store_group<G, F32>(x.p, at + c0 * G, a.ovec, y[0]);
                    store_group<G, F32>(x.p, at + c1 * G, a.ovec, y[1]);
                }
                continue;
            }
            // Float32's z is within 14 u = 14 * 2^-24 of the 64-bit one, relative to the length h
            // of its pair: the sum of squares 9 u (four in a row, three and two levels more), half
            // of which shows in the root, the mean with eps 0.5 u, the root, r w and its product
            // with x 1 u each: 8 u; a product of the two and their sum 2 u; cosine and sine 1 u and
            // 2 pi 2^-26 < 1.6 u of their angle, absolute, for both together 2^0.5 as much of h:
            // 3.7 u.  With the scale's two roundings below 16 u.
            bool sure = true, bad1 = false;
            float near[2] = {0.0f, 0.0f};
            if (in) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if ((c ? c1 : c0) * G >= a.R) {
#pragma unroll
                        for (int e = 0; e < G; ++e) E[c] = fmaxf(E[c], y[c][e] * y[c][e]);
                    }
                    // (the least length: of squares below float32)
                    near[c] = fmaxf(__fsqrt_rn(E[c]), 1e-22f) * ((c ? c1 : c0) * G < a.R ? (float)a.scale : 1.0f) * 0x1p-20f;
                }
                sure = quantise_near<G>(y[0], near[0], w[0], &t[0], &bad);
                sure &= quantise_near<G>(y[1], near[1], w[1], &t[1], &bad1);
                bad |= bad1;
            }
            const uint32_t again = __ballot_sync(0xffffffffu, !sure) & mask;
            if (again) {  // (all four lanes of the row)
                const int g[2] = {c0, c1};
                float z[2 * G], tt[2] = {t[0], t[1]};
                uint32_t ww[2 * (G / 8)];
#pragma unroll
                for (int e = 0; e < 2 * G; ++e) z[e] = y[e / G][e % G];
#pragma unroll
                for (int e = 0; e < 2 * (G / 8); ++e) ww[e] = w[e / (G / 8)][e % (G / 8)];
                exact_groups<D, F32, INTER>(Exact<D, F32, INTER>{a, a.k.p, b * a.k.b + i * a.k.i + h * a.k.h, a.kw, h * a.kw.h, b, i, 1.0}, mask, g, z,
                                            near, ww, tt);
                t[0] = tt[0], t[1] = tt[1];
#pragma unroll
                for (int e = 0; e < 2 * (G / 8); ++e) w[e / (G / 8)][e % (G / 8)] = ww[e];
            }
            if (!in) continue;
        }
        if (!APPEND) continue;
        if (bad) atomicOr(&st[tok], ACES_ROW_NONFINITE);
        if (!ACES_IN(pos, a.S)) continue;
        uint8_t *row = (kind == 2 ? a.cv : a.ck) + ((size_t)((size_t)b * a.H + h) * a.S + (size_t)pos) * RB;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int g = c ? c1 : c0;
            uint32_t *to = reinterpret_cast<uint32_t *>(row) + g * (G / 8);
            if (G == 16)
                *reinterpret_cast<uint2 *>(to) = make_uint2(w[c][0], w[c][G / 8 - 1]);
            else
                *to = w[c][0];
            reinterpret_cast<unsigned short *>(row + D / 2)[g] = (unsigned short)(__float_as_uint(t[c]) >> 16);
        }
    }
    if (APPEND) {
        __syncthreads();
        if (tid < tokens) a.status[(size_t)b * a.n + i0 + tid] = st[tid];
    }
}

// Tokens of a CTA (their logarithm): several once that still gives every SM four CTAs.
static int turn_tokens(const Turn &a, int nsm) {
    int lt = 0;
    while ((2 << lt) <= TOKENS && (long long)a.B * a.n >= (8ll * nsm) << lt) ++lt;
    return lt;
}

template <int D, bool F32, bool APPEND>
static cudaError_t run_turn(const Turn &a, bool interleaved, int nsm, cudaStream_t s) {
    const int lt = turn_tokens(a, nsm);
    const long long grid = (long long)a.B * ((a.n + (1 << lt) - 1) >> lt);
    if (interleaved)
        k_turn<D, F32, APPEND, true><<<(unsigned)grid, TN, 0, s>>>(a, lt);
    else
        k_turn<D, F32, APPEND, false><<<(unsigned)grid, TN, 0, s>>>(a, lt);
    return cudaGetLastError();
}

cudaError_t launch_turn(const Turn &a, int D, bool f32, bool append, bool interleaved, int nsm, cudaStream_t s) {
    if (D == 64) {
        if (append) return f32 ? run_turn<64, true, true>(a, interleaved, nsm, s) : run_turn<64, false, true>(a, interleaved, nsm, s);
        return f32 ? run_turn<64, true, false>(a, interleaved, nsm, s) : run_turn<64, false, false>(a, interleaved, nsm, s);
    }
    if (append) return f32 ? run_turn<128, true, true>(a, interleaved, nsm, s) : run_turn<128, false, true>(a, interleaved, nsm, s);
    return f32 ? run_turn<128, true, false>(a, interleaved, nsm, s) : run_turn<128, false, false>(a, interleaved, nsm, s);
}

#ifdef ACES_CHECKED
cudaError_t check_take_turn(unsigned long long out[3]) { return check_take(out); }
#endif

}  // namespace aces
