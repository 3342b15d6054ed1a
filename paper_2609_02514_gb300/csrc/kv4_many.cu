// Attention over a 4-bit KV cache for many query rows (trees, prompts) of
// bfloat16 (the format: kv4.cuh, the shares: kv4_plan.cuh), on the 5th-generation
// tensor cores.
//
// A persistent CTA an SM works on items of up to 256 query rows, 128 keys a
// tile, with its warps in five parts:
//   - two softmax groups of four warps, a thread a row: each has 128 rows of
//     scores S, of weights P and of sums O in TMEM and its queries in shared
//     memory.  With more than 128 rows the groups have a half each and share
//     the tiles; with up to 128 both have the same rows and every other tile,
//     and are merged at the end.
//   - one warp brings tiles of rows into a ring in shared memory (bulk copies, as a
//     tile's rows lie in one piece);
//   - six warps turn their codes into bfloat16 tiles in shared memory, in
//     the 128-byte swizzle.  Keys and values lie alike ([key][64 channels] a
//     half): the keys' product reads them along the channels, the values' along
//     the keys (the transposed form of the second operand).
//   - one warp issues the products: S = Q K' of a tile (both from shared memory),
//     O += P V of half a tile at a time (P from TMEM, in the place of its half of
//     S).  While one group turns its scores into weights the other's products run.
// The tensor pipe runs products in the order they were issued, so an S may be
// made in the place of a P whose product is under way.
// Sums are rescaled only when a row's maximum grew by more than 2^8 (in the
// weights' scale); weights stay below that and lose nothing by it.  Weights are
// rounded to bfloat16 for their product, as the tensor cores take them: all 24 bits
// would be three products, and half a unit of eight bits is what the result's own
// rounding costs (the sums of weights take them as they were); scores and sums are float32, the sums by the tensor cores for as many keys as
// FOLD allows.
//
// What bounds it is a group's chain (scores out of TMEM, maximum, exponentials,
// weights back in, 64 keys at a time): a tile of 256 rows of 128 takes 4.1 thousand
// cycles, its products alone 2.6, and 45 to 55 of 100 issue slots are taken.  128 keys in
// one product of scores and weights by halves instead of 64 of each: 1003 -> 770 us
// (4096 tokens of two sequences behind 4000, 32 heads over 8).  That call: 740 us,
// 1.09 PFLOP/s; trees of 80 tokens, 16 sequences: 127 us, 0.59; 2048 tokens of four
// sequences behind a window of 1024, 16 heads of 64: 127 us, 0.27.  Beside the
// tiles an item pays for its queries, its pipeline's start and its way out, two to
// four tiles' time, a fifth of the last one's.
#define ACES_FILE 9  // site numbers of the checked build
#include <climits>

#include <cuda_bf16.h>

#include "kv4_plan.cuh"
#include "warp_wait.cuh"

namespace aces {

constexpr int MKT = 128;                  // keys of a tile
constexpr int MKH = 64;                   // keys of a step of weights
constexpr int MSM = 8, MDQ = 6;           // softmax and dequantising warps
constexpr int MLD = MSM + MDQ, MMM = MLD + 1;  // the warp that loads, the one that issues
constexpr int MT = (MMM + 1) * 32;        // 16 warps of 128 registers
constexpr int MDT = MDQ * 32;
// Measured on 152 CTAs, in thousands of cycles: a tile of two groups' rows 4.1 (D =
// 64: 4.4), of one's 2.7; an item 15.5 (D = 64: 10.2).
template <int D>
struct ManyCost {
    static constexpr int FIX = D == 128 ? 23 : 14, MOST = 6;
    static __device__ __forceinline__ int weight(const Kv4Keys &k) { return k.rows <= 128 ? 4 : 6; }
    static __device__ __forceinline__ int all(const Kv4Keys &k) { return FIX + k.units * weight(k); }
};
constexpr float M_LAZY = 8.0f;
// Tiles of a group after which its sums leave TMEM for float32 totals in the workspace:
// the tensor cores' adds (one for 16 keys) cut off up to a unit each, so sums of one sign
// lie up to 2^-13 low then.  Without totals, values of one sign behind 600000 positions
// came out 3.6e-3 low, twice the rounding of the result; with them 1e-4.
constexpr int FOLD = 128;
// -- tcgen05 ------------------------------------------------------------------
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p;
}
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
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(addr));
}
// The loads before it are done.  The numbers pass through it, so nothing that
// uses them comes before.
__device__ __forceinline__ void tc_wait_ld(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                   "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]),
                   "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]),
                   "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
                 :
                 : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t addr, float (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(addr));
}
__device__ __forceinline__ void tc_wait_ld(float (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
                 :
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
// (addr16: address / 16; below 2^14, as shared memory ends at 228 KB)
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr16, uint32_t lead) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(addr16 | (lead >> 4) << 16), "r"((1024u >> 4) | 1u << 14 | 2u << 29));
    return d;
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

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
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
    static constexpr int RAW = MKT * RB, NR = D == 128 ? 3 : 6;  // a tile's keys or values as they are, and how many
    static constexpr int SMEM = 6 * TILE + NR * RAW + 1024;  // queries of two groups, two stages of keys and values
    static constexpr int PIECES = MKT * D / 32;            // 16-byte pieces of a tile's codes
    static constexpr int PC = (PIECES + MDT - 1) / MDT;    // that a thread dequantises (a warp's last may be none)
    static_assert(PIECES % 32 == 0, "whole warps");
    static constexpr int TS = 0, TP = 32, TO = 256;        // TMEM columns: S[group], a half's P in the second half of that half, O[group]
};

// Byte of 16-byte chunk c (eight channels) of a row in a swizzled tile.
__device__ __forceinline__ uint32_t swz(int row, int c) { return (c >> 3) * (MKT * 128) + row * 128 + (((c ^ row) & 7) << 4); }

template <int D>
struct Piece {  // 32 channels of a row and their t's
    uint4 w;
    uint32_t t[D == 128 ? 1 : 2];
};

template <int D>
__device__ __forceinline__ void load_piece(const uint8_t *raw, int p, Piece<D> &o) {
    constexpr int Q = D / 32;
    const int q = p % Q;
    const uint8_t *r = raw + p / Q * Many<D>::RB;
    o.w = reinterpret_cast<const uint4 *>(r)[q];
    if (D == 128) {
        o.t[0] = reinterpret_cast<const uint32_t *>(r + D / 2)[q];
    } else {
        const uint2 v = reinterpret_cast<const uint2 *>(r + D / 2)[q];
        o.t[0] = v.x;
        o.t[D == 128 ? 0 : 1] = v.y;
    }
}

template <int D>
__device__ __forceinline__ void store_piece(uint8_t *tile, int p, const Piece<D> &o) {
    constexpr int Q = D / 32;
    const int row = p / Q, q = p % Q;
    uint32_t w[4] = {o.w.x, o.w.y, o.w.z, o.w.w}, tt[4];
    const uint32_t t0 = o.t[0] & KV4_T_MASK, t1 = o.t[D == 128 ? 0 : 1] & KV4_T_MASK;
    int flip = 0;
    if (D == 128) {
        tt[0] = tt[1] = __byte_perm(t0, 0, 0x1010);
        tt[2] = tt[3] = __byte_perm(t0, 0, 0x3232);
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
        tt[0] = __byte_perm(t0, 0, 0x1010);
        tt[1] = __byte_perm(t0, 0, 0x3232);
        tt[2] = __byte_perm(t1, 0, 0x1010);
        tt[3] = __byte_perm(t1, 0, 0x3232);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t v[4];
        kv4_pairs(w[k], tt[k], kv4_offset(tt[k]), v);
        *reinterpret_cast<uint4 *>(tile + swz(row, q * 4 + (k ^ flip))) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

// Adds a row's sums in TMEM to its totals (256 floats apart, their maximum behind
// them; the first time there are none) and leaves zeros.
template <int D>
static __device__ __noinline__ void fold_sums(float *tot, uint32_t tO, float m, bool first) {
    const float was = first ? -INFINITY : tot[256 * D], keep = was == -INFINITY ? 0.0f : ex2(was - m);
    tot[256 * D] = m;
#pragma unroll 1
    for (int w = 0; w < D / 16; ++w) {
        float o[16];
        uint32_t zero[16];
        tc_ld16(tO + 16 * w, o);
        tc_wait_ld(o);
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            float *to = tot + 256 * (16 * w + c);
            *to = first ? o[c] : fmaf(*to, keep, o[c]);
            zero[c] = 0u;
        }
        tc_st16(tO + 16 * w, zero);
    }
    tc_wait_st();
}

template <int D>
__global__ void __launch_bounds__(MT, 1) k_kv4_many(Kv4Att a, Kv4Ws ws, int R, int RT) {
    using C = Many<D>;
    using Cost = ManyCost<D>;
    using Seg = Kv4Seg<MKT, 1, Cost>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) unsigned long long bars[33];
    __shared__ uint32_t tmem_base;
    __shared__ float sm_m[2][128], sm_l[2][128];
    __shared__ int any_timeout;
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // the same in all lanes, also for the compiler
    // tiles start on 1024 bytes
    uint8_t *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    const uint32_t sm0 = smem_u32(smem);
    uint8_t *sq = smem, *sk = smem + 2 * C::TILE, *sv = smem + 4 * C::TILE, *raw = smem + 6 * C::TILE;
    const uint32_t bar0 = smem_u32(bars);
    // barriers by stage (keys, values), by group, or by group and half (2 x + half)
    const uint32_t b_kfull = bar0, b_kfree = bar0 + 16, b_vfull = bar0 + 32, b_vfree = bar0 + 48, b_o = bar0 + 64, b_q = bar0 + 80,
                   b_s = bar0 + 96, b_f = bar0 + 112, b_p = bar0 + 128, b_end = bar0 + 160, b_rfull = bar0 + 168, b_rfree = bar0 + 216;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_kfull + 8 * i, MDQ);
            mbar_init(b_vfull + 8 * i, MDQ);
            mbar_init(b_kfree + 8 * i, 1);
            mbar_init(b_vfree + 8 * i, 1);
            mbar_init(b_o + 8 * i, 1);
            mbar_init(b_q + 8 * i, 4);
            mbar_init(b_s + 8 * i, 1);
            mbar_init(b_f + 8 * i, 1);
        }
        for (int i = 0; i < 4; ++i) mbar_init(b_p + 8 * i, 4);
        for (int i = 0; i < C::NR; ++i) {
            mbar_init(b_rfull + 8 * i, 1);
            mbar_init(b_rfree + 8 * i, MDQ);
        }
        mbar_init(b_end, 1);
        any_timeout = 0;
    }
    pdl_trigger();  // the join may be placed as CTAs leave; it waits for all of them
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    const Kv4Start at = kv4_start<MKT, 1, Cost, MT>(a, R, RT);
    if (tid == 0) kv4_put_info<Cost>(ws, at);
    Seg seg;
    if (!seg.start(a, R, RT, at)) return;
    if (warp == MMM) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_before();
    }
    __syncthreads();
    tc_after();
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem_base, 0);
    const int NR = a.n * a.G;  // at most 2^30
    bool bad = false;  // a wait gave up: nothing is waited for any more
    auto wait = [&](uint32_t bar, uint32_t phase) {
        if (!bad && !mbar_wait(bar, phase & 1)) bad = true;
    };

    if (warp < MSM) {
        // -- softmax: a thread a row ------------------------------------------
        const int x = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tm + lanes + C::TS + x * 128, tO = tm + lanes + C::TO + x * D;
        uint8_t *myq = sq + x * C::TILE;
        uint32_t n_s = 0, n_o = 0;  // tiles and segments before this one
        bool first = true;
        do {
            const Kv4Keys &key = seg.key;
            const int b = seg.b, rt = seg.rt, h = seg.h, P = key.P;
            const bool single = NR - rt * R <= 128;
            const int slot_row = single ? row : x * 128 + row;
            const int r0 = rt * R + slot_row, i = r0 / a.G, gq = r0 - i * a.G;
            const bool row_live = r0 < NR && key.live && i < key.cnt;
            const int pos = row_live ? kv4_pos(P, a.mask ? a.depth + b * a.depth_b : nullptr, i) : 0;
            const bool warp_live = __any_sync(0xffffffffu, row_live);
            const int posmax = __reduce_max_sync(0xffffffffu, pos), imin = __reduce_min_sync(0xffffffffu, row_live ? i : INT_MAX);
            const int all_see = a.mask || !warp_live ? P : P + imin + 1;
            const int T = min(seg.x1, key.tiles) - seg.x0;  // 0 for an item without keys
            const int mine = 2 * (single ? (T + 1 - x) >> 1 : T);  // of 64 keys
            // Queries (a row without one reads the first token's and keeps zeros), where the
            // group has tiles: it then waits for their products below.  For a segment without
            // any (padding) it waits for nothing, and words for two of those could both be
            // there before the issuing warp looks: it would take the second for none.
            if (mine > 0) {
                const unsigned short *f = reinterpret_cast<const unsigned short *>(a.q) + b * a.qb + (row_live ? i : 0) * a.qi +
                                          (long long)(h * a.G + (row_live ? gq : 0)) * a.qh;
                const uint32_t keep = row_live ? 0xFFFFFFFFu : 0u;
                if (((uintptr_t)f & 15) == 0) {
#pragma unroll 1
                    for (int c0 = 0; c0 < D / 8; c0 += 8) {
                        uint4 w[8];
#pragma unroll
                        for (int c = 0; c < 8; ++c) w[c] = __ldg(reinterpret_cast<const uint4 *>(f) + c0 + c);
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            *reinterpret_cast<uint4 *>(myq + swz(row, c0 + c)) =
                                make_uint4(bf2_poison(w[c].x) & keep, bf2_poison(w[c].y) & keep, bf2_poison(w[c].z) & keep,
                                           bf2_poison(w[c].w) & keep);
                    }
                } else {
#pragma unroll 1
                    for (int c = 0; c < D / 8; ++c) {
                        uint32_t u[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            u[j] = bf2_poison((uint32_t)__ldg(f + 8 * c + 2 * j) | (uint32_t)__ldg(f + 8 * c + 2 * j + 1) << 16) & keep;
                        *reinterpret_cast<uint4 *>(myq + swz(row, c)) = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                }
                async_fence();
                tc_before();  // the last segment's sums are read
                __syncwarp();
                if (lane == 0) mbar_arrive(b_q + 8 * x);
            }
            float m = -INFINITY, l0 = 0.0f, l1 = 0.0f;
            for (int y = 0; y < mine;) {
                if (y > 0) {  // to the totals: the last tile's product is over before these scores are made
                    wait(b_s + 8 * x, n_s);
                    tc_after();
                    if (warp_live) fold_sums<D>(ws.total + (size_t)blockIdx.x * 256 * (D + 1) + x * 128 + row, tO, m, y == 2 * FOLD);
                }
                const int stop = min(mine, y + 2 * FOLD);
#pragma unroll 1
                for (; y < stop; ++y) {
                    const int half = y & 1;
                    if (half == 0) {
                        wait(b_s + 8 * x, n_s);
                        tc_after();
                    }
                    if (warp_live) {
                        const int j0 = kv4_tile<MKT>(key, seg.x0 + (single ? (y & ~1) + x : y >> 1)) + half * MKH;
                        const bool masked = j0 + MKH > all_see || (a.window && j0 <= posmax - a.window && j0 + MKH > a.sinks);
                        const uint32_t at = tS + half * MKH;
                        float v[2][32];
                        tc_ld32(at, v[0]);
                        tc_ld32(at + 32, v[1]);
                        tc_wait_ld(v[0]);
                        tc_wait_ld(v[1]);
                        if (masked) {
                            uint32_t see0 = 0u, see1 = 0u;
                            if (row_live) see0 = seen_word(a, b, P, key.cnt, j0, i, pos), see1 = seen_word(a, b, P, key.cnt, j0 + 32, i, pos);
#pragma unroll
                            for (int c = 0; c < 32; ++c) {
                                if (!(see0 >> c & 1u)) v[0][c] = -INFINITY;
                                if (!(see1 >> c & 1u)) v[1][c] = -INFINITY;
                            }
                            __syncwarp();
                        }
                        float m0 = v[0][0], m1 = v[0][31], m2 = v[1][0], m3 = v[1][31];
#pragma unroll
                        for (int c = 1; c < 15; c += 2) {
                            m0 = max3(m0, v[0][c], v[0][c + 1]), m1 = max3(m1, v[0][c + 15], v[0][c + 16]);
                            m2 = max3(m2, v[1][c], v[1][c + 1]), m3 = max3(m3, v[1][c + 15], v[1][c + 16]);
                        }
                        m0 = max3(m0, v[0][15], v[0][30]), m2 = max3(m2, v[1][15], v[1][30]);
                        const float mx = fmaxf(max3(m0, m1, m2), m3) * a.scale;
                        const bool grew = mx > m + M_LAZY || (m == -INFINITY && mx > m);
                        if (__any_sync(0xffffffffu, grew)) {
                            const float f = grew ? ex2(m - mx) : 1.0f;
                            if (grew) m = mx;
                            l0 *= f, l1 *= f;
                            if (y > 0) {
                                // what was added last is there: before these scores were
                                // made, or (the first half's) by a word of its own
                                if (half == 1) wait(b_f + 8 * x, n_s);
                                tc_after();
#pragma unroll 1
                                for (int w = 0; w < D / 16; ++w) {
                                    float o[16];
                                    tc_ld16(tO + 16 * w, o);
                                    tc_wait_ld(o);
                                    uint32_t u[16];
#pragma unroll
                                    for (int c = 0; c < 16; ++c) u[c] = __float_as_uint(o[c] * f);
                                    tc_st16(tO + 16 * w, u);
                                }
                            }
                        }
                        const float ref = m == -INFINITY ? 0.0f : -m;
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            uint32_t pk[16];
                            float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
                            for (int c = 0; c < 16; ++c) {
                                float *e = v[w] + 2 * c;
                                fma2(e[0], e[1], a.scale, ref);
                                e[0] = ex2(e[0]), e[1] = ex2(e[1]);
                                add2(s0, s1, e[0], e[1]);
                                pk[c] = bf2_pack(e[0], e[1]);
                            }
                            l0 += s0, l1 += s1;
                            tc_st16(at + C::TP + 16 * w, pk);
                        }
                        tc_wait_st();
                    }
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_p + 8 * (2 * x + half));
                    n_s += half;
                }
            }
            if (mine > 0) {
                wait(b_o + 8 * x, n_o++);
                tc_after();
            }
            // results; their places are worked out here, not kept in registers
            // through the loop (behind an asm the compiler cannot see through)
            float l = l0 + l1;
            int srow = slot_row, srt = seg.rt;
            asm volatile("" : "+r"(srow), "+r"(srt));
            const int r = srt * R + srow, ri = r / a.G;
            const bool live = r < NR && seg.key.live && ri < seg.key.cnt;
            const bool whole = seg.whole();
            float *slot = ws.piece + (size_t)(2 * blockIdx.x + (first ? 0 : 1)) * R * (D + 2);
            const int orow = (seg.b * a.n + ri) * a.Hq + seg.h * a.G + (r - ri * a.G);  // at most 2^30
            // what the totals count for, those of the rows' weights being to m
            const bool folded = mine > 2 * FOLD && warp_live;
            const float *tot = ws.total + (size_t)blockIdx.x * 256 * (D + 1) + x * 128 + row;
            float f = 1.0f, ft = 0.0f;
            if (folded && tot[256 * D] != -INFINITY) ft = ex2(tot[256 * D] - m);
            if (single) {  // both groups have the rows
                sm_m[x][row] = m, sm_l[x][row] = l;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                const float M = fmaxf(sm_m[0][row], sm_m[1][row]), ref = M == -INFINITY ? 0.0f : M;
                f = ex2(m - ref);
                l = sm_l[0][row] * ex2(sm_m[0][row] - ref) + sm_l[1][row] * ex2(sm_m[1][row] - ref);
                m = M;
            }
            const float k = whole ? (live && l != 0.0f ? f * KV4_STEP / l : 0.0f) : f;
            // the second group's sums go to the first through its queries' place
            float4 *box = reinterpret_cast<float4 *>(sq + C::TILE);  // 32 channels of 128 rows
#pragma unroll 1
            for (int w = 0; w < D / 32; ++w) {
                float v[32];
                __syncwarp();
                if (mine > 0 && warp_live) {
                    tc_ld32(tO + 32 * w, v);
                    tc_wait_ld(v);
                    if (folded) {
#pragma unroll
                        for (int c = 0; c < 32; ++c) v[c] = fmaf(tot[256 * (32 * w + c)], ft, v[c]);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c) v[c] = 0.0f;
                }
                if (k == 0.0f) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) v[c] = 0.0f;
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c) v[c] *= k;
                }
                if (single) {
                    if (x == 1) {
#pragma unroll
                        for (int c = 0; c < 8; ++c) box[c * 128 + row] = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
                    }
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    if (x == 0) {
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            const float4 o = box[c * 128 + row];
                            v[4 * c] += o.x, v[4 * c + 1] += o.y, v[4 * c + 2] += o.z, v[4 * c + 3] += o.w;
                        }
                    }
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    if (x == 1) continue;
                }
                // The warp's rows go out in whole lines, through the place of its
                // queries: bfloat16 rows at once, float32 pieces half a row at a time.
                constexpr int CH = D / 8;  // 16-byte chunks of a row there
                // (each warp in its own rows' place: another may be at the next segment's queries)
                auto chunk = [&](int rw, int c) { return reinterpret_cast<uint4 *>(myq + swz(rw, c)); };
                bool full;
                if (whole) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        *chunk(row, 4 * w + c) = make_uint4(bf2_pack(v[8 * c], v[8 * c + 1]), bf2_pack(v[8 * c + 2], v[8 * c + 3]),
                                                            bf2_pack(v[8 * c + 4], v[8 * c + 5]), bf2_pack(v[8 * c + 6], v[8 * c + 7]));
                    full = w == D / 32 - 1;
                } else {
                    const int c0 = (w % (D / 64)) * 8;
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        *chunk(row, c0 + c) = make_uint4(__float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]),
                                                         __float_as_uint(v[4 * c + 2]), __float_as_uint(v[4 * c + 3]));
                    full = w % (D / 64) == D / 64 - 1;
                }
                if (!full) continue;
                __syncwarp();
                const int r_first = r - lane, rw0 = row - lane, sw0 = srow - lane;
#pragma unroll 4
                for (int z = 0; z < CH; ++z) {  // 32 / CH rows at a time
                    const int rr = z * (32 / CH) + lane / CH, c = lane % CH;
                    const int to = __shfl_sync(0xffffffffu, orow, rr);
                    if (r_first + rr >= NR) continue;
                    const uint4 o = *chunk(rw0 + rr, c);
                    if (whole)
                        reinterpret_cast<uint4 *>(a.out)[(size_t)to * CH + c] = o;
                    else
                        reinterpret_cast<uint4 *>(slot)[(size_t)(sw0 + rr) * (D / 4) + (w / (D / 64)) * CH + c] = o;
                }
                __syncwarp();
            }
            if (r < NR && !(single && x == 1)) {
                if (!whole) {
                    slot[(size_t)R * D + srow] = m;
                    slot[(size_t)R * D + R + srow] = l;
                } else if (a.lse) {
                    a.lse[orow] = live && l != 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
                }
            }
            first = false;
        } while (seg.next(a, R, RT));
    } else if (warp < MSM + MDQ) {
        // -- codes to bfloat16 tiles ------------------------------------------
        const int dt = tid - MSM * 32;
        uint32_t step = 0;  // 2 x the tile's number (+ 1: its values)
        do {
            const int T = min(seg.x1, seg.key.tiles) - seg.x0;
#pragma unroll 1
            for (int y = 0; y < 2 * T; ++y, ++step) {
                const uint32_t st = (step >> 1) & 1, v = step & 1, rs = step % C::NR;
                Piece<D> p[C::PC];
                wait(b_rfull + 8 * rs, step / C::NR);
#pragma unroll
                for (int u = 0; u < C::PC; ++u)
                    if (dt + u * MDT < C::PIECES) load_piece<D>(raw + rs * C::RAW, dt + u * MDT, p[u]);
                wait((v ? b_vfree : b_kfree) + 8 * st, (step >> 2) + 1);
                uint8_t *tile = (v ? sv : sk) + st * C::TILE;
#pragma unroll
                for (int u = 0; u < C::PC; ++u)
                    if (dt + u * MDT < C::PIECES) store_piece<D>(tile, dt + u * MDT, p[u]);
                async_fence();
                __syncwarp();
                // The rows' place is given back only here: the next copy into it is not
                // ordered after loads that are still under way.
                if (lane == 0) {
                    mbar_arrive((v ? b_vfull : b_kfull) + 8 * st);
                    mbar_arrive(b_rfree + 8 * rs);
                }
            }
        } while (seg.next(a, R, RT));
    } else if (warp == MLD) {
        // -- rows into the ring: keys, values, keys ... -----------------------
        if (lane == 0) {
            // Rows are asked into the L2 AHEAD tiles before they are loaded: memory's
            // latency at its full rate is more than the ring holds.
            constexpr int AHEAD = 6;
            const uint32_t raw0 = smem_u32(raw);
            uint32_t step = 0;
            do {
                const uint8_t *kb = a.k + seg.row0(a) * C::RB, *vb = a.v + seg.row0(a) * C::RB;  // the key head's rows
                const int top = min(seg.x1, seg.key.tiles), end = seg.key.P + seg.key.cnt;
                int ahead = seg.x0 + 1;
#pragma unroll 1
                for (int y = seg.x0; y < top && !bad; ++y) {
                    for (; ahead < min(top, y + AHEAD); ++ahead) {
                        const int j0 = kv4_tile<MKT>(seg.key, ahead);
                        const uint32_t bytes = min(MKT, end - j0) * C::RB;
                        const unsigned long long off = (unsigned long long)(uint32_t)j0 * (uint32_t)C::RB;
                        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(kb + off), "r"(bytes) : "memory");
                        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(vb + off), "r"(bytes) : "memory");
                    }
                    const int j0 = kv4_tile<MKT>(seg.key, y);
                    // past the sequence's end the ring keeps what it has: any bytes are
                    // numbers, and their weights are 0
                    const uint32_t bytes = min(MKT, end - j0) * C::RB;
                    const unsigned long long off = (unsigned long long)(uint32_t)j0 * (uint32_t)C::RB;
                    const bool in = ACES_IN(j0, a.S) && ACES_IN(end - 1, a.S);
#pragma unroll 1
                    for (int v = 0; v < 2; ++v, ++step) {
                        const uint32_t rs = step % C::NR;
                        wait(b_rfree + 8 * rs, step / C::NR + 1);
                        if (bad) break;
                        mbar_expect(b_rfull + 8 * rs, in ? bytes : 0);
                        if (in) bulk_load(raw0 + rs * C::RAW, (v ? vb : kb) + off, bytes, b_rfull + 8 * rs);
                    }
                }
            } while (!bad && seg.next(a, R, RT));
            // no copy is under way when the CTA ends, also after a wait that gave up
            for (uint32_t z = step > C::NR ? step - C::NR : 0; z < step; ++z)
                if (!mbar_wait(b_rfull + 8 * (z % C::NR), (z / C::NR) & 1)) bad = true;
        }
    } else {
        // -- products: the whole warp goes along, so that addresses stay in uniform
        // registers, and one lane issues -------------------------------------
        const uint32_t q0 = sm0, k0 = sm0 + 2 * C::TILE, v0 = sm0 + 4 * C::TILE;
        constexpr uint32_t ID_S = tc_idesc(MKT, false), ID_O = tc_idesc(D, true);
        const bool leader = elect_one();
        auto go = [&](uint32_t bar, uint32_t phase) {  // wait(), with one answer for the warp
            if (bad) return;
            bad = !warp_wait([&] { return mbar_try(bar, phase & 1); }, [&] { return mbar_wait_slow(bar, phase & 1); },
                             [](bool ok) { return (bool)__all_sync(0xffffffffu, ok); });
        };
        uint32_t n = 0, n0 = 0, n1 = 0, q0s = 0, q1s = 0;  // tiles, each group's tiles and its queries so far
        do {
            const bool single = NR - seg.rt * R <= 128;
            const int T = __shfl_sync(0xffffffffu, min(seg.x1, seg.key.tiles) - seg.x0, 0);
            const int cnt0 = single ? (T + 1) >> 1 : T, cnt1 = single ? T >> 1 : T;
            if (cnt0 > 0) go(b_q, q0s++);
            if (cnt1 > 0) go(b_q + 8, q1s++);
            // each group in turn: the values of its tile i, then the scores of i + 1
#pragma unroll 1
            for (int u = -2; u < 2 * cnt0 && !bad; ++u) {
                const int x = u & 1, i = u >> 1, mine = x ? cnt1 : cnt0;  // i from -1
                const uint32_t ts = tm + C::TS + x * MKT;
                const bool first = single || x == 0, last = single || x == 1;  // of a tile's users
                if (i >= 0 && i < mine) {
                    const uint32_t tile = n + (single ? 2 * i + x : i), st = tile & 1, ph = (x ? n1 : n0) + i;
                    const uint32_t bd = (v0 + st * C::TILE) >> 4, to = tm + C::TO + x * D;
                    if (first) go(b_vfull + 8 * st, tile >> 1);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        go(b_p + 8 * (2 * x + half), ph);
                        tc_after();
                        if (leader && !bad) {
#pragma unroll
                            for (int ks = 0; ks < MKH / 16; ++ks)
                                tc_mma_ts(to, ts + half * MKH + C::TP + 8 * ks, tc_desc(bd + (half * (MKH / 16) + ks) * (2048 >> 4), C::HALF),
                                          ID_O, i > 0 || half > 0 || ks > 0);
                            if (half == 0) tc_commit(b_f + 8 * x);
                        }
                    }
                    if (leader && !bad) {
                        if (last) tc_commit(b_vfree + 8 * st);
                        if (i + 1 == mine) tc_commit(b_o + 8 * x);
                    }
                }
                if (i + 1 < mine) {
                    const uint32_t tile = n + (single ? 2 * (i + 1) + x : i + 1), st = tile & 1;
                    if (first) go(b_kfull + 8 * st, tile >> 1);
                    const uint32_t ad = (q0 + x * C::TILE) >> 4, bd = (k0 + st * C::TILE) >> 4;
                    if (leader && !bad) {
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks) {
                            const uint32_t o = ((ks >> 2) * C::HALF + (ks & 3) * 32) >> 4;
                            tc_mma_ss(ts, tc_desc(ad + o, 16), tc_desc(bd + o, 16), ID_S, ks > 0);
                        }
                        tc_commit(b_s + 8 * x);
                        if (last) tc_commit(b_kfree + 8 * st);
                    }
                }
                __syncwarp();
            }
            n += max(T, 0);
            n0 += max(cnt0, 0), n1 += max(cnt1, 0);
        } while (seg.next(a, R, RT));
        if (leader) tc_commit(b_end);  // nothing runs on when the columns are given back
        if (!mbar_wait(b_end, 0)) bad = true;
    }
    if (bad) any_timeout = 1;
    __syncwarp();
    tc_before();
    __syncthreads();
    if (tid == 0 && any_timeout) ws.info[blockIdx.x].timeout = 1;
    if (warp == MMM) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm) : "memory");
    }
}

// Rows of an item.
static int many_rows_of(int n, int G) { return (long long)n * G <= 128 ? 128 : 256; }

// (after the pieces: a CTA's totals, [D] by 256 rows and their maximum)
size_t kv4_many_ws(int n, int G, int D, int nsm) { return kv4_ws_bytes(nsm, many_rows_of(n, G), D) + (size_t)nsm * 256 * (D + 1) * 4; }

template <int D>
static cudaError_t run_many(const Kv4Att &a, void *workspace, int nsm, cudaStream_t s) {
    const int R = many_rows_of(a.n, a.G), RT = (int)(((long long)a.n * a.G + R - 1) / R);
    Kv4Ws ws = kv4_ws_carve(workspace, nsm);
    ws.total = ws.piece + (size_t)2 * nsm * R * (D + 2);
    static std::atomic<unsigned long long> allowed{0};
    cudaError_t e = allow_smem(k_kv4_many<D>, Many<D>::SMEM, allowed);
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
