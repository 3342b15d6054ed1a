// Attention over a 4-bit KV cache for many query rows (trees, prompts) of
// bfloat16 (the format: kv4.cuh, the shares: kv4_plan.cuh), on the 5th-generation
// tensor cores.
//
// A persistent CTA an SM works on items of up to 256 query rows, 128 keys a
// tile, with its warps in four parts:
//   - two softmax groups of four warps, a thread a row: each has 128 rows of
//     scores S, of weights P and of sums O in TMEM and its queries in shared
//     memory.  With more than 128 rows the groups have a half each and share
//     the tiles; with up to 128 both have the same rows and every other tile,
//     and are merged at the end.
//   - eight warps turn the rows' codes into bfloat16 tiles in shared memory, in
//     the 128-byte swizzle.  Keys and values lie alike ([key][64 channels] a
//     half): the keys' product reads them along the channels, the values' along
//     the keys (the transposed form of the second operand).
//   - one thread issues the products: S = Q K' (both from shared memory), O += P
//     V (P from TMEM).  While one group turns its scores into weights the
//     other's products run.
// P takes the place of S (D = 128): the products of both have one shape, so the
// tensor pipe runs them in the order they were issued.  For D = 64 the shapes
// differ and P has columns of its own.
// Sums are rescaled only when a row's maximum grew by more than 2^8 (in the
// weights' scale); weights stay below that and lose nothing by it.
#define ACES_FILE 9  // site numbers of the checked build
#include <climits>

#include <cuda_bf16.h>

#include "kv4_plan.cuh"

namespace aces {

constexpr int MKT = 128;                  // keys of a tile
constexpr int MSM = 8, MDQ = 8;           // softmax and dequantising warps
constexpr int MT = (MSM + MDQ + 1) * 32;  // and the one that issues
constexpr int MDT = MDQ * 32;
constexpr float M_LAZY = 8.0f;

// -- tcgen05 ------------------------------------------------------------------
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
// 32 columns of this warp's 32 rows
__device__ __forceinline__ void tc_ld32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tc_st32(uint32_t addr, const float (&v)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"f"(v[0]),
        "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]),
        "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]),
        "f"(v[22]), "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31]),
        "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(v[0]),
        "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
        "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(addr)
        : "memory");
}

// Shared-memory descriptor of the 128-byte swizzle: eight rows of 128 bytes are
// 1024 bytes apart from the next eight (stride); lead: the next 64 channels of
// an operand read along the keys.
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr, uint32_t lead) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// kind::f16: float32 sums of bfloat16, M = 128, N, second operand along N
__host__ __device__ constexpr uint32_t tc_idesc(int N, bool b_mn) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (b_mn ? 1u << 16 : 0u) | (uint32_t)(N >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
}

// two float32 at once
__device__ __forceinline__ void fma2(float &x, float &y, float a, float c) {
    asm("{\n\t.reg .b64 u, v, w;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %2};\n\tmov.b64 w, {%3, %3};\n\t"
        "fma.rn.f32x2 u, u, v, w;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(x), "+f"(y)
        : "f"(a), "f"(c));
}
__device__ __forceinline__ void add2(float &x, float &y, float a, float b) {
    asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tadd.rn.f32x2 u, u, v;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(x), "+f"(y)
        : "f"(a), "f"(b));
}

// bits [lo, hi) of the word of positions [w0, w0 + 32)
__device__ __forceinline__ uint32_t span_bits(int lo, int hi, int w0) {
    const int x = max(lo - w0, 0), y = min(hi - w0, 32);
    if (x >= y) return 0u;
    return (y >= 32 ? 0xFFFFFFFFu : (1u << y) - 1u) & ~((1u << x) - 1u);
}
// Which of the positions [w0, w0 + 32) token i at position pos sees.
__device__ __forceinline__ uint32_t seen_word(const Kv4Att &a, int b, int P, int cnt, int w0, int i, int pos) {
    const int first = a.window ? pos - a.window + 1 : 0;
    if (!a.mask) return span_bits(0, P + i + 1, w0) & (span_bits(first, INT_MAX, w0) | span_bits(0, a.sinks, w0));
    uint32_t r = w0 < P ? span_bits(0, P, w0) & (span_bits(first, INT_MAX, w0) | span_bits(0, a.sinks, w0)) : 0u;
    if (w0 + 32 <= P || w0 >= P + cnt) return r;
    const uint32_t *row = a.mask + b * a.mask_b + (size_t)i * a.words;
    const int t0 = w0 - P;  // the token at w0, above -32
    const int wi = t0 >> 5, sh = t0 & 31;
    const uint32_t lo = wi >= 0 ? __ldg(row + wi) : 0u, hi = wi + 1 < a.words ? __ldg(row + wi + 1) : 0u;
    uint32_t bits = __funnelshift_r(lo, hi, sh) & span_bits(P, P + cnt, w0);
    if (a.window && a.window <= pos - P) {  // some new tokens may lie behind the window
        const int32_t *dep = a.depth + b * a.depth_b;
        for (uint32_t left = bits; left; left &= left - 1) {
            const int x = __ffs(left) - 1, kp = kv4_pos(P, dep, t0 + x);
            if (kp < first && kp >= a.sinks) bits &= ~(1u << x);
        }
    }
    return r | bits;
}

template <int D>
struct Many {
    static constexpr int RB = kv4_row_bytes(D);
    static constexpr int HALF = MKT * 128;                 // 128 rows of 64 channels
    static constexpr int TILE = MKT * D * 2;
    static constexpr int SMEM = 6 * TILE + 1024;           // queries of two groups, two stages of keys and values
    static constexpr int PC = MKT * D / 32 / MDT;          // 16-byte pieces a thread dequantises of a tile
    static constexpr int TS = 0, TO = 256, TP = D == 128 ? 0 : 384, TPX = D == 128 ? 128 : 64;  // TMEM columns
};

// Byte of 16-byte chunk c (eight channels) of a row in a swizzled tile.
__device__ __forceinline__ uint32_t swz(int row, int c) { return (c >> 3) * (MKT * 128) + row * 128 + (((c ^ row) & 7) << 4); }

template <int D>
struct Piece {  // 32 channels of a row and their t's
    uint4 w;
    uint32_t t[D == 128 ? 1 : 2];
};

template <int D>
__device__ __forceinline__ void load_piece(const uint8_t *plane, size_t row0, int j0, int end, int p, Piece<D> &o) {
    constexpr int RB = Many<D>::RB, Q = D / 32;
    const int row = p / Q, q = p % Q;
    o.w = make_uint4(0u, 0u, 0u, 0u);
    o.t[0] = 0u;
    if (D == 64) o.t[D == 128 ? 0 : 1] = 0u;
    if (j0 + row >= end) return;  // past the sequence: zeros
    const uint8_t *r = plane + (row0 + j0 + row) * RB;
    o.w = __ldg(reinterpret_cast<const uint4 *>(r) + q);
    if (D == 128) {
        o.t[0] = __ldg(reinterpret_cast<const uint32_t *>(r + D / 2) + q) & KV4_T_MASK;
    } else {
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(r + D / 2) + q);
        o.t[0] = v.x & KV4_T_MASK;
        o.t[D == 128 ? 0 : 1] = v.y & KV4_T_MASK;
    }
}

template <int D>
__device__ __forceinline__ void store_piece(uint8_t *tile, int p, const Piece<D> &o) {
    constexpr int Q = D / 32;
    const int row = p / Q, q = p % Q;
    uint32_t w[4] = {o.w.x, o.w.y, o.w.z, o.w.w}, tt[4];
    int flip = 0;
    if (D == 128) {
        tt[0] = tt[1] = __byte_perm(o.t[0], 0, 0x1010);
        tt[2] = tt[3] = __byte_perm(o.t[0], 0, 0x3232);
        // eight lanes have two rows; the rows' upper halves, 16 KB further, fall on
        // the same banks, so they go in another order
        flip = q & 2;
        if (flip) {
            uint32_t x;
            x = w[0], w[0] = w[2], w[2] = x;
            x = w[1], w[1] = w[3], w[3] = x;
            x = tt[0], tt[0] = tt[1] = tt[2], tt[2] = tt[3] = x;
        }
    } else {
        tt[0] = __byte_perm(o.t[0], 0, 0x1010);
        tt[1] = __byte_perm(o.t[0], 0, 0x3232);
        tt[2] = __byte_perm(o.t[D == 128 ? 0 : 1], 0, 0x1010);
        tt[3] = __byte_perm(o.t[D == 128 ? 0 : 1], 0, 0x3232);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t v[4];
        kv4_pairs(w[k], tt[k], kv4_offset(tt[k]), v);
        *reinterpret_cast<uint4 *>(tile + swz(row, q * 4 + (k ^ flip))) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

template <int D>
__global__ void __launch_bounds__(MT, 1) k_kv4_many(Kv4Att a, Kv4Ws ws, int R, int RT) {
    using C = Many<D>;
    using Seg = Kv4Seg<MKT, 1>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) unsigned long long bars[17];
    __shared__ uint32_t tmem_base;
    __shared__ float sm_m[2][128], sm_l[2][128];
    __shared__ int any_timeout;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // tiles start on 1024 bytes
    uint8_t *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    const uint32_t sm0 = smem_u32(smem);
    uint8_t *sq = smem, *sk = smem + 2 * C::TILE, *sv = smem + 4 * C::TILE;
    const uint32_t bar0 = smem_u32(bars);
    // pairs of barriers by stage (keys, values) or by group
    const uint32_t b_kfull = bar0, b_kfree = bar0 + 16, b_vfull = bar0 + 32, b_vfree = bar0 + 48, b_s = bar0 + 64, b_p = bar0 + 80,
                   b_o = bar0 + 96, b_q = bar0 + 112, b_end = bar0 + 128;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_kfull + 8 * i, MDQ);
            mbar_init(b_vfull + 8 * i, MDQ);
            mbar_init(b_kfree + 8 * i, 1);
            mbar_init(b_vfree + 8 * i, 1);
            mbar_init(b_s + 8 * i, 1);
            mbar_init(b_o + 8 * i, 1);
            mbar_init(b_p + 8 * i, 4);
            mbar_init(b_q + 8 * i, 4);
        }
        mbar_init(b_end, 1);
        any_timeout = 0;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    const Kv4Start at = kv4_start<MKT, 1, MT>(a, R, RT);
    if (tid == 0) kv4_put_info<MKT, 1>(a, ws, at, R, RT);
    Seg seg;
    if (!seg.start(a, R, RT, at)) return;
    if (warp == MSM + MDQ) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_before();
    }
    __syncthreads();
    tc_after();
    const uint32_t tm = tmem_base;
    const long long NR = (long long)a.n * a.G;
    bool bad = false;  // a wait gave up: nothing is waited for any more
    auto wait = [&](uint32_t bar, uint32_t phase) {
        if (!bad && !mbar_wait(bar, phase & 1)) bad = true;
    };

    if (warp < MSM) {
        // -- softmax: a thread a row ------------------------------------------
        const int x = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tm + lanes + C::TS + x * 128, tO = tm + lanes + C::TO + x * D, tP = tm + lanes + C::TP + x * C::TPX;
        uint8_t *myq = sq + x * C::TILE;
        uint32_t n_s = 0, n_o = 0;  // phases passed
        bool first = true;
        do {
            const Kv4Keys &key = seg.key;
            const int b = seg.e / RT, rt = seg.e % RT, h = seg.h, P = key.P;
            const bool single = NR - (long long)rt * R <= 128;
            const int slot_row = single ? row : x * 128 + row;
            const long long r = (long long)rt * R + slot_row;
            const int i = (int)(r / a.G), gq = (int)(r % a.G);
            const bool live = r < NR && key.live && i < key.cnt;
            const int pos = live ? kv4_pos(P, a.mask ? a.depth + b * a.depth_b : nullptr, i) : 0;
            const bool warp_live = __any_sync(0xffffffffu, live);
            const int posmax = __reduce_max_sync(0xffffffffu, pos), imin = __reduce_min_sync(0xffffffffu, live ? i : INT_MAX);
            const int all_see = a.mask || !warp_live ? P : P + imin + 1;
            const int T = min(seg.x1, key.tiles) - seg.x0;  // 0 for an item without keys
            const int mine = single ? (T + 1 - x) >> 1 : T;
            // queries
            {
                const unsigned short *f = reinterpret_cast<const unsigned short *>(a.q) + b * a.qb + i * a.qi + (long long)(h * a.G + gq) * a.qh;
                const bool vec = ((uintptr_t)f & 15) == 0;
#pragma unroll 4
                for (int c = 0; c < D / 8; ++c) {
                    uint4 w = make_uint4(0u, 0u, 0u, 0u);
                    if (live) {
                        if (vec) {
                            w = __ldg(reinterpret_cast<const uint4 *>(f) + c);
                        } else {
                            uint32_t u[4];
                            for (int j = 0; j < 4; ++j) u[j] = (uint32_t)__ldg(f + 8 * c + 2 * j) | (uint32_t)__ldg(f + 8 * c + 2 * j + 1) << 16;
                            w = make_uint4(u[0], u[1], u[2], u[3]);
                        }
                        w.x = bf2_poison(w.x), w.y = bf2_poison(w.y), w.z = bf2_poison(w.z), w.w = bf2_poison(w.w);
                    }
                    *reinterpret_cast<uint4 *>(myq + swz(row, c)) = w;
                }
            }
            async_fence();
            tc_before();  // the last segment's sums are read
            __syncwarp();
            if (lane == 0) mbar_arrive(b_q + 8 * x);
            float m = -INFINITY, l0 = 0.0f, l1 = 0.0f;
            for (int y = 0; y < mine; ++y) {
                wait(b_s + 8 * x, n_s++);
                tc_after();
                if (warp_live) {
                    const int j0 = kv4_tile<MKT>(key, seg.x0 + (single ? 2 * y + x : y));
                    const bool masked = j0 + MKT > all_see || (a.window && j0 <= posmax - a.window && j0 + MKT > a.sinks);
                    uint32_t seen[4] = {0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu};
                    if (masked) {
#pragma unroll
                        for (int w = 0; w < 4; ++w) seen[w] = live ? seen_word(a, b, P, key.cnt, j0 + 32 * w, i, pos) : 0u;
                    }
                    __syncwarp();
                    float mx = -INFINITY;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        float v[32];
                        tc_ld32(tS + 32 * w, v);
                        tc_wait_ld();
                        if (masked) {
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (!(seen[w] >> c & 1u)) v[c] = -INFINITY;
                        }
                        float m0 = v[0], m1 = v[1];
#pragma unroll
                        for (int c = 2; c < 32; c += 2) m0 = fmaxf(m0, v[c]), m1 = fmaxf(m1, v[c + 1]);
                        mx = fmaxf(mx, fmaxf(m0, m1));
                    }
                    mx *= a.scale;
                    const bool grew = mx > m + M_LAZY || (m == -INFINITY && mx > m);
                    if (__any_sync(0xffffffffu, grew)) {
                        const float f = grew ? ex2(m - mx) : 1.0f;
                        if (grew) m = mx;
                        l0 *= f, l1 *= f;
                        if (y > 0) {
#pragma unroll
                            for (int w = 0; w < D / 32; ++w) {
                                float v[32];
                                tc_ld32(tO + 32 * w, v);
                                tc_wait_ld();
#pragma unroll
                                for (int c = 0; c < 32; ++c) v[c] *= f;
                                tc_st32(tO + 32 * w, v);
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.0f : -m;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        float v[32];
                        tc_ld32(tS + 32 * w, v);
                        tc_wait_ld();
                        if (masked) {
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (!(seen[w] >> c & 1u)) v[c] = -INFINITY;
                        }
                        uint32_t pk[16];
#pragma unroll
                        for (int c = 0; c < 16; ++c) {
                            fma2(v[2 * c], v[2 * c + 1], a.scale, ref);
                            v[2 * c] = ex2(v[2 * c]), v[2 * c + 1] = ex2(v[2 * c + 1]);
                            add2(l0, l1, v[2 * c], v[2 * c + 1]);
                            pk[c] = bf2_pack(v[2 * c], v[2 * c + 1]);
                        }
                        tc_st16(tP + 16 * w, pk);
                    }
                    tc_wait_st();
                }
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_p + 8 * x);
            }
            if (mine > 0) {
                wait(b_o + 8 * x, n_o++);
                tc_after();
            }
            // results
            float l = l0 + l1;
            const bool whole = seg.whole();
            float *slot = ws.piece + (size_t)(2 * blockIdx.x + (first ? 0 : 1)) * R * (D + 2);
            const size_t orow = ((size_t)b * a.n + i) * a.Hq + h * a.G + gq;
            auto put = [&](int w, const float (&v)[32]) {  // channels 32 w ..
                if (r >= NR) return;
                if (whole) {
                    const float k = live && l != 0.0f ? KV4_STEP / l : 0.0f;
                    uint4 *o = reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(a.out) + orow * D + 32 * w);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t u[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) u[j] = k == 0.0f ? 0u : bf2_pack(v[8 * c + 2 * j] * k, v[8 * c + 2 * j + 1] * k);
                        o[c] = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                } else {
                    float4 *o = reinterpret_cast<float4 *>(slot + (size_t)slot_row * D + 32 * w);
#pragma unroll
                    for (int c = 0; c < 8; ++c) o[c] = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
                }
            };
            auto put_stats = [&]() {
                if (r >= NR) return;
                if (whole) {
                    if (a.lse) a.lse[orow] = live && l != 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
                } else {
                    slot[(size_t)R * D + slot_row] = m;
                    slot[(size_t)R * D + R + slot_row] = l;
                }
            };
            auto sums = [&](int w, float (&v)[32]) {
                __syncwarp();
                if (mine > 0 && warp_live) {
                    tc_ld32(tO + 32 * w, v);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c) v[c] = 0.0f;
                }
            };
            if (!single) {
#pragma unroll 1
                for (int w = 0; w < D / 32; ++w) {
                    float v[32];
                    sums(w, v);
                    put(w, v);
                }
                put_stats();
            } else {
                // the second group's sums go to the first through its queries' place
                sm_m[x][row] = m, sm_l[x][row] = l;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                const float M = fmaxf(sm_m[0][row], sm_m[1][row]), ref2 = M == -INFINITY ? 0.0f : M, f = ex2(m - ref2);
                l = sm_l[0][row] * ex2(sm_m[0][row] - ref2) + sm_l[1][row] * ex2(sm_m[1][row] - ref2);
                m = M;
                float4 *box = reinterpret_cast<float4 *>(sq + C::TILE);  // D / 2 channels of 128 rows
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    if (x == 1) {
#pragma unroll 1
                        for (int w = 0; w < D / 64; ++w) {
                            float v[32];
                            sums(half * (D / 64) + w, v);
#pragma unroll
                            for (int c = 0; c < 8; ++c)
                                box[(w * 8 + c) * 128 + row] = make_float4(v[4 * c] * f, v[4 * c + 1] * f, v[4 * c + 2] * f, v[4 * c + 3] * f);
                        }
                    }
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    if (x == 0) {
#pragma unroll 1
                        for (int w = 0; w < D / 64; ++w) {
                            float v[32];
                            sums(half * (D / 64) + w, v);
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const float4 o = box[(w * 8 + c) * 128 + row];
                                v[4 * c] = fmaf(v[4 * c], f, o.x), v[4 * c + 1] = fmaf(v[4 * c + 1], f, o.y);
                                v[4 * c + 2] = fmaf(v[4 * c + 2], f, o.z), v[4 * c + 3] = fmaf(v[4 * c + 3], f, o.w);
                            }
                            put(half * (D / 64) + w, v);
                        }
                    }
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                }
                if (x == 0) put_stats();
            }
            first = false;
        } while (seg.next(a, R, RT));
    } else if (warp < MSM + MDQ) {
        // -- codes to bfloat16 tiles ------------------------------------------
        const int dt = tid - MSM * 32;
        uint32_t n = 0;  // tiles done
        Seg pre = seg;   // what is asked into the L2 ahead of the loads
        int py = pre.x0;
        bool pmore = dt == 0;
        auto prefetch = [&]() {
            while (pmore && py >= min(pre.x1, pre.key.tiles)) {
                pmore = pre.next(a, R, RT);
                py = pre.x0;
            }
            if (!pmore) return;
            const int j0 = kv4_tile<MKT>(pre.key, py++), rows = min(MKT, pre.key.P + pre.key.cnt - j0);
            const size_t off = ((size_t)((size_t)(pre.e / RT) * a.H + pre.h) * a.S + j0) * C::RB;
            const uint32_t bytes = rows * C::RB;
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.k + off), "r"(bytes) : "memory");
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.v + off), "r"(bytes) : "memory");
        };
        Piece<D> pk[C::PC], pv[C::PC];
        int y = seg.x0;
        bool more = true;
        auto settle = [&]() {  // y: the next tile there is
            while (more && y >= min(seg.x1, seg.key.tiles)) {
                more = seg.next(a, R, RT);
                y = seg.x0;
            }
        };
        auto load = [&](const uint8_t *plane, Piece<D> (&p)[C::PC]) {
            const int j0 = kv4_tile<MKT>(seg.key, y), end = seg.key.P + seg.key.cnt;
            const size_t row0 = (size_t)((size_t)(seg.e / RT) * a.H + seg.h) * a.S;
            if (!ACES_IN(j0, a.S) || !ACES_IN(end - 1, a.S)) return;
#pragma unroll
            for (int u = 0; u < C::PC; ++u) load_piece<D>(plane, row0, j0, end, dt + u * MDT, p[u]);
        };
        for (int u = 0; u < 6; ++u) prefetch();
        settle();
        if (more) {
            load(a.k, pk);
            load(a.v, pv);
        }
        while (more) {
            const uint32_t st = n & 1, ph = n >> 1;
            prefetch();
            wait(b_kfree + 8 * st, ph + 1);
#pragma unroll
            for (int u = 0; u < C::PC; ++u) store_piece<D>(sk + st * C::TILE, dt + u * MDT, pk[u]);
            async_fence();
            __syncwarp();
            if (lane == 0) mbar_arrive(b_kfull + 8 * st);
            ++y;
            settle();
            if (more) load(a.k, pk);
            wait(b_vfree + 8 * st, ph + 1);
#pragma unroll
            for (int u = 0; u < C::PC; ++u) store_piece<D>(sv + st * C::TILE, dt + u * MDT, pv[u]);
            async_fence();
            __syncwarp();
            if (lane == 0) mbar_arrive(b_vfull + 8 * st);
            if (more) load(a.v, pv);
            ++n;
        }
    } else if (lane == 0) {
        // -- products ---------------------------------------------------------
        const uint32_t q0 = sm0, k0 = sm0 + 2 * C::TILE, v0 = sm0 + 4 * C::TILE;
        constexpr uint32_t ID_S = tc_idesc(MKT, false), ID_O = tc_idesc(D, true);
        uint32_t n = 0, segs = 0, n_p[2] = {0, 0};
        do {
            const int rt = seg.e % RT;
            const bool single = NR - (long long)rt * R <= 128;
            const int T = min(seg.x1, seg.key.tiles) - seg.x0;
            int cnt[2];
            cnt[0] = single ? (T + 1) >> 1 : T;
            cnt[1] = single ? T >> 1 : T;
            auto scores = [&](int x, int i) {
                const uint32_t tile = n + (single ? 2 * i + x : i), st = tile & 1;
                wait(b_kfull + 8 * st, tile >> 1);
                if (bad) return;
                tc_after();
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t o = (ks >> 2) * C::HALF + (ks & 3) * 32;
                    tc_mma_ss(tm + C::TS + x * 128, tc_desc(q0 + x * C::TILE + o, 16), tc_desc(k0 + st * C::TILE + o, 16), ID_S, ks > 0);
                }
                tc_commit(b_s + 8 * x);
                if (single || x == 1) tc_commit(b_kfree + 8 * st);
            };
            auto values = [&](int x, int i) {
                const uint32_t tile = n + (single ? 2 * i + x : i), st = tile & 1;
                wait(b_vfull + 8 * st, tile >> 1);
                wait(b_p + 8 * x, n_p[x]++);
                if (bad) return;
                tc_after();
#pragma unroll
                for (int ks = 0; ks < MKT / 16; ++ks)
                    tc_mma_ts(tm + C::TO + x * D, tm + C::TP + x * C::TPX + 8 * ks, tc_desc(v0 + st * C::TILE + ks * 2048, C::HALF), ID_O,
                              i > 0 || ks > 0);
                if (single || x == 1) tc_commit(b_vfree + 8 * st);
                if (i + 1 == cnt[x]) tc_commit(b_o + 8 * x);
            };
            wait(b_q, segs);
            if (cnt[0] > 0) scores(0, 0);
            wait(b_q + 8, segs);
            if (cnt[1] > 0) scores(1, 0);
            for (int i = 0; i < cnt[0]; ++i) {
                values(0, i);
                if (i + 1 < cnt[0]) scores(0, i + 1);
                if (i < cnt[1]) {
                    values(1, i);
                    if (i + 1 < cnt[1]) scores(1, i + 1);
                }
            }
            n += max(T, 0);
            ++segs;
        } while (seg.next(a, R, RT));
        tc_commit(b_end);  // nothing runs on when the columns are given back
        if (!mbar_wait(b_end, 0)) bad = true;
    }
    if (bad) any_timeout = 1;
    __syncwarp();
    tc_before();
    __syncthreads();
    if (tid == 0 && any_timeout) ws.info[blockIdx.x].timeout = 1;
    if (warp == MSM + MDQ) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm) : "memory");
    }
}

// Rows of an item.
static int many_rows_of(int n, int G) { return (long long)n * G <= 128 ? 128 : 256; }

size_t kv4_many_ws(int n, int G, int D, int nsm) { return kv4_ws_bytes(nsm, many_rows_of(n, G), D); }

template <int D>
static cudaError_t run_many(const Kv4Att &a, void *workspace, int nsm, cudaStream_t s) {
    const int R = many_rows_of(a.n, a.G), RT = (int)(((long long)a.n * a.G + R - 1) / R);
    const Kv4Ws ws = kv4_ws_carve(workspace, nsm);
    cudaError_t e = cudaFuncSetAttribute(k_kv4_many<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Many<D>::SMEM);
    if (e != cudaSuccess) return e;
    k_kv4_many<D><<<nsm, MT, Many<D>::SMEM, s>>>(a, ws, R, RT);
    e = cudaGetLastError();
    return e != cudaSuccess ? e : launch_kv4_join(a, ws, nsm, R, s);
}

cudaError_t launch_kv4_many(const Kv4Att &a, void *workspace, int nsm, cudaStream_t s) {
    return a.D == 64 ? run_many<64>(a, workspace, nsm, s) : run_many<128>(a, workspace, nsm, s);
}

#ifdef ACES_CHECKED
cudaError_t check_take_kv4_many(unsigned long long out[3]) { return check_take(out); }
#endif

}  // namespace aces
