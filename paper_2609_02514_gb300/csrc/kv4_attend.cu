// Attention over a 4-bit KV cache (the format: kv4.cuh): one CTA a query row.
//
// The CTA takes 128 keys a step with a running maximum and sum: a thread
// multiplies its key with the query, then takes one channel (D = 64: half the
// keys of one) of the weighted values.
#define ACES_FILE 8  // site numbers of the checked build
#include <cuda_bf16.h>
#include <math_constants.h>

#include "kv4.cuh"

namespace aces {

constexpr int NTA = 128;

__device__ __forceinline__ float kv4_at(const uint8_t *row, int D, int d) {
    const uint32_t w = __ldg(reinterpret_cast<const uint32_t *>(row) + d / 8);
    const int e = d % 8;
    const uint32_t t = __ldg(reinterpret_cast<const unsigned short *>(row + D / 2) + d / (D / 8)) & 0xBFFFu;
    return (float)((int)((w >> (4 * (e >> 1) + 16 * (e & 1))) & 15u) - 8) * __uint_as_float(t << 16);
}

template <int D, bool F32>
__global__ void __launch_bounds__(NTA) k_kv4_rows(Kv4Att a) {
    constexpr int RB = kv4_row_bytes(D), SPL = NTA / D;
    __shared__ float q[D], p[NTA], red[NTA / 32], acc[NTA];
    const int hq = blockIdx.x % a.Hq, i = (blockIdx.x / a.Hq) % a.n, b = blockIdx.x / (a.Hq * a.n);
    const int tid = threadIdx.x, h = hq / a.G;
    const Kv4Seq sq = kv4_seq(a.prefix, a.count, b, a.n, a.S);
    if (i == 0 && hq == 0 && tid == 0) a.status[b] = sq.ok ? 0 : ACES_ROW_RANGE;
    const size_t orow = ((size_t)b * a.n + i) * a.Hq + hq;
    const bool live = sq.ok && i < sq.cnt;
    if (tid < D) {
        const long long at = b * a.qb + i * a.qi + hq * a.qh + tid;
        if (F32) q[tid] = __ldg(reinterpret_cast<const float *>(a.q) + at);
        if (!F32) q[tid] = __uint_as_float((uint32_t)__ldg(reinterpret_cast<const unsigned short *>(a.q) + at) << 16);
    }
    __syncthreads();
    const uint32_t *mrow = a.mask ? a.mask + b * a.mask_b + (size_t)i * a.words : nullptr;
    const int32_t *dep = a.mask ? a.depth + b * a.depth_b : nullptr;
    const int pos = kv4_pos(sq.P, dep, i);
    const int end = !live ? 0 : sq.P + (a.mask ? sq.cnt : i + 1);
    const int lo = a.window ? max(0, min(pos, sq.P) - a.window + 1) : 0;
    const uint8_t *kr = a.k + ((size_t)b * a.H + h) * a.S * RB, *vr = a.v + ((size_t)b * a.H + h) * a.S * RB;
    float m = -INFINITY, l = 0.0f, o = 0.0f;
    for (int j0 = 0; j0 < end; j0 += NTA) {
        if (a.window && j0 >= a.sinks && j0 + NTA <= lo) continue;
        const int j = j0 + tid;
        float s = -INFINITY;
        if (j < end) {
            bool vis = true;
            int kp = j;
            if (j >= sq.P && mrow) {
                const int t = j - sq.P;
                vis = (mrow[t >> 5] >> (t & 31)) & 1u;
                kp = kv4_pos(sq.P, dep, t);
            }
            if (a.window) vis = vis && (kp > pos - a.window || kp < a.sinks);
            if (vis) {
                s = 0.0f;
                for (int d = 0; d < D; ++d) s = fmaf(q[d], kv4_at(kr + (size_t)j * RB, D, d), s);
                s *= a.scale;
            }
        }
        float mx = warp_max(s);
        __syncthreads();
        if ((tid & 31) == 0) red[tid >> 5] = mx;
        __syncthreads();
        for (int w = 0; w < NTA / 32; ++w) mx = fmaxf(mx, red[w]);
        const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.0f : mn;
        const float e = ex2(s - ref), f = ex2(m - ref);
        l = l * f + e;
        o *= f;
        m = mn;
        p[tid] = e;
        __syncthreads();
        const int top = min(NTA, end - j0);
        for (int x = tid / D; x < top; x += SPL) o = fmaf(p[x], kv4_at(vr + (size_t)(j0 + x) * RB, D, tid % D), o);
    }
    acc[tid] = o;
    for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
    __syncthreads();
    if ((tid & 31) == 0) red[tid >> 5] = l;
    __syncthreads();
    l = 0.0f;
    for (int w = 0; w < NTA / 32; ++w) l += red[w];
    if (tid < D) {
        for (int x = 1; x < SPL; ++x) o += acc[tid + x * D];
        const float r = l > 0.0f || l != l ? o * KV4_STEP / l : 0.0f;
        if (F32)
            reinterpret_cast<float *>(a.out)[orow * D + tid] = r;
        else
            reinterpret_cast<__nv_bfloat16 *>(a.out)[orow * D + tid] = __float2bfloat16_rn(r);
    }
    if (tid == 0 && a.lse) a.lse[orow] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

size_t kv4_attention_ws(int B, int n, int Hq, int H, int D) { return 16; }

cudaError_t launch_kv4_attention(const Kv4Att &a, void *workspace, cudaStream_t s) {
    (void)workspace;
    const unsigned grid = (unsigned)((long long)a.B * a.n * a.Hq);
    if (a.D == 64)
        a.f32 ? k_kv4_rows<64, true><<<grid, NTA, 0, s>>>(a) : k_kv4_rows<64, false><<<grid, NTA, 0, s>>>(a);
    else
        a.f32 ? k_kv4_rows<128, true><<<grid, NTA, 0, s>>>(a) : k_kv4_rows<128, false><<<grid, NTA, 0, s>>>(a);
    return cudaGetLastError();
}

#ifdef ACES_CHECKED
cudaError_t check_take_kv4_attend(unsigned long long out[3]) { return check_take(out); }
#endif

}  // namespace aces
