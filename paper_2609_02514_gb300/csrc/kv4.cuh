// The rows of a 4-bit KV cache, and what its kernels share.
//
// A row holds one head's D numbers of one position (D = 64 or 128) in
// D / 2 + 16 bytes: D / 8 words of eight 4-bit codes, then eight bfloat16
// numbers t, one for each group of D / 8 consecutive channels.  Channel
// 8 i + 2 j lies at bits 4 j of word i, channel 8 i + 2 j + 1 at bits 16 + 4 j.
//
//   step  s = t * 2^16, t = -a * 2^-19 rounded to five significant bits (ties
//         to even), a the group's first number of largest magnitude;
//   value (c - 8) * s with the code c = clamp(rint(x / s), -8, 7) + 8.
//
// The sign of s puts a on -8, the longer arm of the codes.  c - 8 has three
// significant bits and s five, so every value is exact in bfloat16: products
// with it on the tensor cores round nothing.  t is below 2 in magnitude; its
// readers clear the exponent bit that says otherwise, so whatever bytes lie in
// a row nobody wrote, they stand for finite numbers, and a masked key's
// probability of 0 times them is 0.  A row is a multiple of 16 bytes, so
// aces_compact_kv moves rows as they are.
#pragma once
#include "common.cuh"

namespace aces {

constexpr int KV4_GROUPS = 8;
constexpr int KV4_PARAM_BYTES = 16;                 // eight bfloat16
constexpr float KV4_STEP = 65536.0f;                // s / t
constexpr float KV4_CAP = 15.5f * 65536.0f;         // largest magnitude held
constexpr float KV4_TINY = 8.077935669463161e-28f;  // 2^-90: a group below it is zeros
constexpr uint32_t KV4_T_MASK = 0xBFFFBFFFu;        // of two t's: magnitudes below 2

__host__ __device__ constexpr int kv4_row_bytes(int D) { return D / 2 + KV4_PARAM_BYTES; }

// t of a group from its number of largest magnitude, |a| <= KV4_CAP
__device__ __forceinline__ float kv4_t(float a) {
    if (!(fabsf(a) >= KV4_TINY)) return 0.0f;
    const uint32_t u = __float_as_uint(a * -1.9073486328125e-06f);  // -2^-19
    uint32_t m = u & 0x7FFFFFFFu;
    m = (m + 0x3FFFFu + ((m >> 19) & 1u)) & ~0x7FFFFu;
    return __uint_as_float((u & 0x80000000u) | m);
}

// x / s as a whole number r (inv: 1 / s; h: |s| / 2; a step of 0: 0 and infinity), in
// the bits of 1.5 * 2^23 + r: no conversions, which run at a quarter of the rate,
// and a word of codes is the sum of the bits, shifted, and KV4_BITS.  |x| is at most
// 8.25 |s|, and above 8 |s| only on the side of -8, so only the other end is cut.
//   bfloat16 x: the quotient after one Newton step is exact where it can be held,
//   and a half can; any other is further from a half than that step's error.
//   float32 x: the estimate may be a little off; the rest d = x - r s is exact (r s
//   has at most nine bits, and d lies on x's grid below |x| or is x), so it
//   decides, on a half to even.
template <bool F32>
__device__ __forceinline__ uint32_t kv4_round(float x, float s, float inv, float h) {
    constexpr float BIG = 12582912.0f;
    float e;
    if (F32) {
        e = fmaf(x, inv, BIG);
        const float d = fmaf(BIG - e, s, x);
        const float one = __uint_as_float(0x3F800000u | ((__float_as_uint(d) ^ __float_as_uint(s)) & 0x80000000u));
        if (fabsf(d) > h || (fabsf(d) == h && (__float_as_uint(e) & 1u))) e += one;
    } else {
        const float q = x * inv;
        e = fmaf(fmaf(-q, s, x), inv, q) + BIG;
    }
    return __float_as_uint(fminf(e, BIG + 7.0f));
}
// turns the bits 0x4B400000 + r into the code r + 8, at each of a word's eight places
constexpr uint32_t KV4_BITS = (8u - 0x4B400000u) * 0x11111111u;

// The number of a sequence's cached positions and of its new ones.
struct Kv4Seq {
    int P, cnt;
    bool ok;
    int shared;  // positions of its prefix (KV4_BEHIND, KV4_SPLIT)
};
__device__ __forceinline__ Kv4Seq kv4_seq(const int32_t *prefix, const int32_t *count, int b, int n, int S) {
    Kv4Seq q;
    q.P = prefix[b];
    q.cnt = count ? count[b] : n;
    q.ok = q.P >= 0 && q.cnt >= 0 && q.cnt <= n && (long long)q.P + q.cnt <= S;
    return q;
}

// What a pass of the attention is: a call of its own, or one of the two of a batch whose
// sequences share prefixes.  The first takes a prefix for a sequence and all tokens of
// those that share it (its group) for its new tokens, which see nothing but the prefix;
// it leaves its sums, not yet divided, with their maximum and the sum of their weights.
// The second takes each sequence's own rows, and adds those sums as one more piece.  Or
// one pass has every sequence's rows in two places, its prefix's tiles before its own.
enum { KV4_ALONE = 0, KV4_FIRST = 1, KV4_BEHIND = 2, KV4_SPLIT = 3 };

// Position of new token t: its depth in the tree (a negative or absurd one is
// taken as the nearest sensible one), or its number.
__device__ __forceinline__ int kv4_pos(int P, const int32_t *depth, int t) {
    return P + (depth ? min(max(depth[t], 0), 1 << 29) : t);
}

// Arguments of the attention kernels.
struct Kv4Att {
    const uint8_t *k, *v;  // the layer's planes [B, H, S, row]
    const void *q;
    long long qb, qi, qh;  // strides of q's sequences, tokens and heads, in elements
    int f32;               // q and out are float32 (else bfloat16)
    void *out;             // [B, n, Hq, D]
    float *lse;            // [B, n, Hq] or null
    int32_t *status;       // [B]
    const int32_t *prefix, *count;
    const uint32_t *mask;  // [n, words] or [B, n, words] or null (causal)
    long long mask_b;      // words between two sequences' masks (0: shared)
    const int32_t *depth;  // [n] or [B, n]; with mask
    long long depth_b;
    int B, n, Hq, H, G, S, D, words;
    int window, sinks;     // window 0: none
    float scale;           // of q . k, in log2 units, times KV4_STEP
    // of two passes: sequences of a group; the first pass's sums [B, n, Hq, D], maxima
    // and sums of weights [B, n, Hq], and status [groups]
    int per;
    float *part, *part_m, *part_l;
    int32_t *part_status;
    const int32_t *shared_len;  // [groups]
    int shared_S;
    const uint8_t *k0, *v0;     // KV4_SPLIT: the prefixes' planes [groups, H, shared_S, row]
    int longest_first;          // CTAs take the sequences by their lengths
    // the first pass: a sequence's tokens (n is a group's), its own positions and counts
    int own_n, own_S;
    const int32_t *own_prefix, *own_count;
};

struct Kv4Rows {
    uint8_t *k, *v;                        // the layer's planes
    void *xk, *xv;                         // [B, n, H, D] numbers
    long long kb, ki, kh, vb, vi, vh;      // their strides in elements
    int f32, vec;                          // vec: every group starts on 16 bytes
    const int32_t *start, *count;
    int32_t *status;                       // [B, n] (append)
    int B, n, H, S, D;
};
cudaError_t launch_kv4_append(const Kv4Rows &a, int nsm, cudaStream_t s);
cudaError_t launch_kv4_read(const Kv4Rows &a, int nsm, cudaStream_t s);

}  // namespace aces
