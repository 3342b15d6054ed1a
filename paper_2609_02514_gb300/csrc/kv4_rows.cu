// Writing a 4-bit KV cache and reading it back (the format: kv4.cuh).
//
// One thread takes one group of a row (8 or 16 channels): its maximum, its
// step and its codes need no other thread.  A CTA takes a few tokens of one
// sequence with all their heads, keys and values, so one store of a token's
// status follows; within a CTA the tokens of one head are neighbours, whose
// cache rows are too.  What a large call has to do is to move numbers on one side
// and 5/8 (D = 128) or 3/4 of a byte each on the other.  Reading does so at 6.4
// TB/s (704.6 MB in 109.9 us).  Writing is 18 (bfloat16) to 43 (float32)
// instructions a number and a few waves of CTAs, each a start and one or two loads'
// way from memory and back: 80 tokens of 64 sequences (eight heads of 128, bfloat16)
// 11.5 us, three waves of 608 CTAs, the last of 64, with two groups a thread, the
// second's load behind the first's store; 4099 of 3 (four of 64, float32) 12.3 us, five
// waves of 760, the last of 35.  Half the issue slots are taken while CTAs run.
#define ACES_FILE 7  // site numbers of the checked build
#include "kv4.cuh"

namespace aces {

constexpr int NT4 = 256;

template <int G, bool F32>
__device__ __forceinline__ void load_group(const void *base, long long at, bool vec, float (&x)[G]) {
    if (F32) {
        const float *p = reinterpret_cast<const float *>(base) + at;
        if (vec) {
#pragma unroll
            for (int i = 0; i < G / 4; ++i) {
                const uint4 w = ldg16(p + 4 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[4 * i + j] = Elem<ACES_F32>::get(w, j);
            }
        } else {
#pragma unroll
            for (int i = 0; i < G; ++i) x[i] = __ldg(p + i);
        }
    } else {
        const unsigned short *p = reinterpret_cast<const unsigned short *>(base) + at;
        if (vec) {
#pragma unroll
            for (int i = 0; i < G / 8; ++i) {
                const uint4 w = ldg16(p + 8 * i);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[8 * i + j] = Elem<ACES_BF16>::get(w, j);
            }
        } else {
#pragma unroll
            for (int i = 0; i < G; ++i) x[i] = __uint_as_float((uint32_t)__ldg(p + i) << 16);
        }
    }
}

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

template <int D, bool F32>
__global__ void __launch_bounds__(NT4) k_kv4_append(Kv4Rows a, int lt) {
    constexpr int G = D / KV4_GROUPS, RB = kv4_row_bytes(D);
    __shared__ int st[8];
    const int T = 1 << lt, per = (a.n + T - 1) >> lt;  // CTAs of a sequence
    const int b = blockIdx.x / per, i0 = (blockIdx.x - b * per) * T;
    const int start = a.start[b], cnt = a.count ? a.count[b] : a.n;
    if (threadIdx.x < T) st[threadIdx.x] = 0;
    __syncthreads();
    const int total = 2 * a.H * T * KV4_GROUPS;
    for (int x = threadIdx.x; x < total; x += NT4) {
        const int g = x % KV4_GROUPS, r = x / KV4_GROUPS;
        const int tok = r & (T - 1), ph = r >> lt, plane = ph >= a.H, h = ph - plane * a.H;
        const int i = i0 + tok;
        if (i >= a.n || i >= cnt) continue;
        const long long pos = (long long)start + i;
        if (pos < 0 || pos >= a.S) {
            if (g == 0) atomicOr(&st[tok], ACES_ROW_RANGE);
            continue;
        }
        float v[G], t;
        uint32_t w[G / 8];
        bool bad;
        const long long at = plane ? b * a.vb + i * a.vi + h * a.vh : b * a.kb + i * a.ki + h * a.kh;
        load_group<G, F32>(plane ? a.xv : a.xk, at + g * G, a.vec, v);
        quantise<G, F32>(v, w, &t, &bad);
        if (bad) atomicOr(&st[tok], ACES_ROW_NONFINITE);
        if (!ACES_IN(pos, a.S)) continue;
        uint8_t *row = (plane ? a.v : a.k) + ((size_t)((size_t)b * a.H + h) * a.S + (size_t)pos) * RB;
        uint32_t *c = reinterpret_cast<uint32_t *>(row) + g * (G / 8);
        if (G == 16)
            *reinterpret_cast<uint2 *>(c) = make_uint2(w[0], w[G / 8 - 1]);
        else
            *c = w[0];
        reinterpret_cast<unsigned short *>(row + D / 2)[g] = (unsigned short)(__float_as_uint(t) >> 16);
    }
    __syncthreads();
    if (threadIdx.x < T && i0 + (int)threadIdx.x < a.n) a.status[(size_t)b * a.n + i0 + threadIdx.x] = st[threadIdx.x];
}

template <int D, bool F32>
__global__ void __launch_bounds__(NT4) k_kv4_read(Kv4Rows a, int lt) {
    constexpr int G = D / KV4_GROUPS, RB = kv4_row_bytes(D);
    const int T = 1 << lt, per = (a.n + T - 1) >> lt;
    const int b = blockIdx.x / per, i0 = (blockIdx.x - b * per) * T;
    const int start = a.start[b];
    const int total = 2 * a.H * T * KV4_GROUPS;
    for (int x = threadIdx.x; x < total; x += NT4) {
        const int g = x % KV4_GROUPS, r = x / KV4_GROUPS;
        const int tok = r & (T - 1), ph = r >> lt, plane = ph >= a.H, h = ph - plane * a.H;
        const int i = i0 + tok;
        if (i >= a.n) continue;
        const long long pos = (long long)start + i;
        uint32_t w[G / 8];
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < G / 8; ++j) w[j] = 0x88888888u;
        if (pos >= 0 && pos < a.S && ACES_IN(pos, a.S)) {
            const uint8_t *row = (plane ? a.v : a.k) + ((size_t)((size_t)b * a.H + h) * a.S + (size_t)pos) * RB;
            const uint32_t *c = reinterpret_cast<const uint32_t *>(row) + g * (G / 8);
#pragma unroll
            for (int j = 0; j < G / 8; ++j) w[j] = __ldg(c + j);
            const uint32_t t = __ldg(reinterpret_cast<const unsigned short *>(row + D / 2) + g) & (KV4_T_MASK & 0xFFFFu);
            s = __uint_as_float(t << 16) * KV4_STEP;
        }
        float v[G];
#pragma unroll
        for (int e = 0; e < G; ++e)
            v[e] = (float)((int)((w[e / 8] >> (4 * ((e % 8) >> 1) + 16 * (e & 1))) & 15u) - 8) * s;
        const size_t at = (((size_t)b * a.n + i) * a.H + h) * D + g * G;
        if (F32) {
            float *o = reinterpret_cast<float *>(plane ? a.xv : a.xk) + at;
#pragma unroll
            for (int j = 0; j < G / 4; ++j)
                *reinterpret_cast<float4 *>(o + 4 * j) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        } else {
            unsigned short *o = reinterpret_cast<unsigned short *>(plane ? a.xv : a.xk) + at;
#pragma unroll
            for (int j = 0; j < G / 8; ++j) {
                uint32_t p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)  // exact: the upper halves
                    p[e] = (__float_as_uint(v[8 * j + 2 * e]) >> 16) | (__float_as_uint(v[8 * j + 2 * e + 1]) & 0xFFFF0000u);
                *reinterpret_cast<uint4 *>(o + 8 * j) = make_uint4(p[0], p[1], p[2], p[3]);
            }
        }
    }
}

// Tokens of a CTA (their logarithm): several neighbours, whose rows of 80 or 48 bytes
// lie side by side, once that still gives every SM four CTAs, else one.  Eight when
// reading (16384 tokens of 8 sequences, eight heads of 128: 109.9 us, by fours
// 114.4), four when writing (80 tokens of 64 sequences: 11.5 us, by eights 12.7, one
// at a time 16.4; 4099 of 3, float32, four heads of 64: 12.3, 12.1, 28.4).
static int tokens_per_cta(const Kv4Rows &a, int lt, int nsm) {
    return (long long)a.B * a.n >= (4ll * nsm) << lt ? lt : 0;
}

template <bool APPEND>
static cudaError_t launch_rows(const Kv4Rows &a, int nsm, cudaStream_t s) {
    const int lt = tokens_per_cta(a, APPEND ? 2 : 3, nsm);
    const long long grid = (long long)a.B * ((a.n + (1 << lt) - 1) >> lt);
    void (*fn)(Kv4Rows, int) = nullptr;
    if (APPEND)
        fn = a.D == 64 ? (a.f32 ? k_kv4_append<64, true> : k_kv4_append<64, false>)
                       : (a.f32 ? k_kv4_append<128, true> : k_kv4_append<128, false>);
    else
        fn = a.D == 64 ? (a.f32 ? k_kv4_read<64, true> : k_kv4_read<64, false>)
                       : (a.f32 ? k_kv4_read<128, true> : k_kv4_read<128, false>);
    fn<<<(unsigned)grid, NT4, 0, s>>>(a, lt);
    return cudaGetLastError();
}

cudaError_t launch_kv4_append(const Kv4Rows &a, int nsm, cudaStream_t s) { return launch_rows<true>(a, nsm, s); }
cudaError_t launch_kv4_read(const Kv4Rows &a, int nsm, cudaStream_t s) { return launch_rows<false>(a, nsm, s); }

#ifdef ACES_CHECKED
cudaError_t check_take_kv4_rows(unsigned long long out[3]) { return check_take(out); }
#endif

}  // namespace aces
