// Attention over a 4-bit KV cache for few query rows (the format: kv4.cuh, the
// shares: kv4_plan.cuh): single tokens, and everything in float32.
#define ACES_FILE 8  // site numbers of the checked build
#include <atomic>

#include <cuda_bf16.h>

#include "kv4_plan.cuh"

namespace aces {

constexpr int FW = 8;            // warps
constexpr int FT = FW * 32;
constexpr int FKT = 32;          // keys of a tile: one warp's step
// Measured on 304 CTAs of ragged single tokens: 3.4 thousand cycles a unit (eight
// tiles), 9.5 thousand an item.
struct FewCost {
    static constexpr int FIX = 3, MOST = 1;
    static __device__ __forceinline__ int weight(const Kv4Keys &) { return 1; }
    static __device__ __forceinline__ int all(const Kv4Keys &k) { return FIX + k.units; }
};
constexpr float F_LAZY = 8.0f;

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
    return d;
}

// -- clusters -----------------------------------------------------------------
constexpr int FCL = 8;  // CTAs of one, at most
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_map(uint32_t addr, int rank) {  // the same place in another CTA
    uint32_t d;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(addr), "r"(rank));
    return d;
}
__device__ __forceinline__ float cluster_ld(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 cluster_ld4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// A wait that gave up: the ring's other copies (a place without one costs as long a wait)
template <int ST>
static __device__ __noinline__ void mbar_drain(uint32_t bar0, int seq) {
    for (int z = seq; z < seq + ST; ++z) mbar_wait_slow(bar0 + 8 * (z % ST), (z / ST) & 1);
}

template <int D, bool F32, int NT>
struct Few {
    static constexpr int RB = kv4_row_bytes(D), R = 8 * NT, KS = D / 16, JT = D / 16, WPT = D / 32;
    static constexpr int SPL = F32 ? 3 : 1;                 // bfloat16 parts of a query number and of a weight
    static constexpr int MINB = !F32 && NT == 1 ? 2 : 1;    // CTAs an SM
    static constexpr int ST = MINB == 2 ? 2 : 4;            // stages of a warp's ring
    static constexpr bool QREG = !F32 && NT == 1;
    static constexpr int STAGE = 2 * FKT * RB, RING = FW * ST * STAGE;
    static constexpr int MERGE = FW * JT * 4 * 32 * 4;
    static constexpr int QS = QREG ? 0 : NT * SPL * KS * 32 * 8;
    static constexpr int SMEM = RING + MERGE + QS;
};

// The tiles stay in registers and shared memory: a warp takes 32 keys at a
// time through a ring of its own (one bulk copy of the keys' rows, one of the
// values'), dequantises them straight into the first operand of the tensor
// products and keeps 8 NT query rows as the second, so no query row is padded
// beyond eight:
//   S' [16 keys x 8 rows] = K [16 x 16 channels] Q',
//   O' [16 channels x 8 rows] += V' [16 x 16 keys] P'.
// A thread's key words are neighbours of one row, its value words the same
// channels of neighbouring keys: channels and keys come in whatever order the
// words have, the same in both operands.  P' needs its pairs along the keys,
// where S' has them along the rows: movmatrix turns the 8 x 8 blocks.
// With bfloat16 queries the weights are rounded to bfloat16 for their product (half a
// unit of eight bits, what the result's own rounding costs; all 24 bits would be three
// products), and the tensor cores add a warp's eighth of the keys up, an add for 16 of
// them, which cuts off up to a unit: 1e-4 for 131072 positions that one CTA has alone.
// Float32 queries and weights are three bfloat16 parts each, all 24 bits.
//
// Most of its time is the codes' way into operands: some 780 warp instructions 32 keys
// of 128, 60 of 100 issue slots taken (and of the ALU's).  One token, 32 heads over 8:
// 32 sequences of 32768 positions 260 us, 5.16 TB/s; 64 of 200 to 8191 88 us, 4.0; one
// of 131071 48 us, 3.5.  The rest of the shorter ones is a CTA's start (3 us: its share,
// its first copies), its warps' merge (2.5 us an item) and the join.  mma.sync and not
// the tcgen05 kernel: its rows are padded to 128 (the rule in kv4_abi.cu).
template <int D, bool F32, int NT>
__global__ void __launch_bounds__(FT, (Few<D, F32, NT>::MINB)) k_kv4_few(Kv4Att a, Kv4Ws ws, int RT, int CL) {
    using C = Few<D, F32, NT>;
    constexpr int RB = C::RB, R = C::R, KS = C::KS, JT = C::JT, WPT = C::WPT, ST = C::ST, SPL = C::SPL;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) unsigned long long bars[FW * ST];
    __shared__ float sm_m[FW][R], sm_l[FW][R];
    __shared__ int2 rowinfo[2][R];              // token and position of a row, of this segment and the next
    __shared__ int any_timeout;
    float *merge = reinterpret_cast<float *>(smem + C::RING);
    uint2 *qs = reinterpret_cast<uint2 *>(smem + C::RING + C::MERGE);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const uint32_t ring = smem_u32(smem) + warp * ST * C::STAGE;
    const uint8_t *ringp = smem + warp * ST * C::STAGE;
    const uint32_t bar0 = smem_u32(bars) + warp * ST * 8;
    if (lane == 0)
        for (int s = 0; s < ST; ++s) mbar_init(bar0 + 8 * s, 1);
    if (tid == 0) any_timeout = 0;
    const bool direct = CL > 0;  // clusters of CL CTAs an item, else shares
    if (!direct) pdl_trigger();  // the join may be placed as CTAs leave; it waits for all of them
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");

    using Seg = Kv4Seg<FKT, FW, FewCost>;
    const Kv4Start at = direct ? kv4_whole<FKT, FW, FewCost>(a, R, RT, CL) : kv4_start<FKT, FW, FewCost, FT>(a, R, RT);
    if (tid == 0 && !direct) kv4_put_info<FewCost>(ws, at);
    __syncwarp();  // each warp waits on its own barriers only
    Seg cur;
    if (!cur.start(a, R, RT, at)) return;
    const int rank = CL > 1 ? blockIdx.x % CL : 0;
    if (CL > 1) cur.x0 = cur.key.units * rank / CL, cur.x1 = cur.key.units * (rank + 1) / CL;

    int seq = 0;       // tiles this warp has taken, of all segments
    bool bad = false;  // a wait gave up
    // this warp's y-th tile of the segment, into the ring's next place
    const uint8_t *kb = nullptr, *vb = nullptr;  // the key head's rows
    auto place_rows = [&](const Seg &g) { kb = a.k + g.row0(a) * RB, vb = a.v + g.row0(a) * RB; };
    place_rows(cur);
    auto issue = [&](const Seg &g, int y, int place) {
        if (lane != 0 || bad) return;
        const int j0 = kv4_tile<FKT>(g.key, (g.x0 + y) * FW + warp), rows = min(FKT, g.key.P + g.key.cnt - j0);
        if (!ACES_IN(j0, a.S) || !ACES_IN(j0 + rows - 1, a.S)) return;
        const int s = place % ST;
        const uint32_t bytes = rows * RB, dst = ring + s * C::STAGE;
        const unsigned long long off = (unsigned long long)(uint32_t)j0 * (uint32_t)RB;
        mbar_expect(bar0 + 8 * s, 2 * bytes);
        bulk_load(dst, kb + off, bytes, bar0 + 8 * s);
        bulk_load(dst + FKT * RB, vb + off, bytes, bar0 + 8 * s);
    };
    auto my_tiles = [&](const Seg &g) {
        const int top = min(g.x1 * FW, g.key.tiles) - g.x0 * FW - warp;
        return top > 0 ? (top + FW - 1) / FW : 0;
    };
    // Eight channels of a query row, part sp of three (float32: 24 bits in parts of
    // eight).  A row that is none reads the first one's and becomes zeros, so the
    // loads need no branch and are all under way at once.
    const bool q_vec = !F32 && (((uintptr_t)a.q | (uintptr_t)(2 * a.qb) | (uintptr_t)(2 * a.qi) | (uintptr_t)(2 * a.qh)) & 15) == 0;
    auto q_at = [&](const Seg &sg, int row, int word, bool &ok) {
        const int r = sg.rt * R + row, ri = r / a.G;
        ok = r < a.n * a.G && sg.key.live && ri < sg.key.cnt;
        const int i = ok ? ri : 0, gq = ok ? r - ri * a.G : 0;
        return sg.b * a.qb + i * a.qi + (long long)(sg.h * a.G + gq) * a.qh + 8 * word;
    };
    auto q_load = [&](const Seg &sg, int row, int word, uint32_t (&o)[4]) {  // bfloat16, as they are
        bool ok;
        const unsigned short *f = reinterpret_cast<const unsigned short *>(a.q) + q_at(sg, row, word, ok);
        if (q_vec) {
            const uint4 w = ldg16(f);
            o[0] = w.x, o[1] = w.y, o[2] = w.z, o[3] = w.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = (uint32_t)__ldg(f + 2 * j) | (uint32_t)__ldg(f + 2 * j + 1) << 16;
        }
    };
    auto q_words = [&](const Seg &sg, int row, int word, int sp, uint32_t (&o)[4]) {
        bool ok;
        const long long p = q_at(sg, row, word, ok);
        if (F32) {
            const float *f = reinterpret_cast<const float *>(a.q) + p;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __ldg(f + j);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // cut off, not rounded: the largest float32 would become infinities
                float v0 = v[2 * j], v1 = v[2 * j + 1];
                uint32_t w = __byte_perm(__float_as_uint(v0), __float_as_uint(v1), 0x7632);
                for (int x = 0; x < sp; ++x) {
                    v0 -= bf_lo(w), v1 -= bf_hi(w);
                    w = __byte_perm(__float_as_uint(v0), __float_as_uint(v1), 0x7632);
                }
                o[j] = w;
            }
        } else {
            q_load(sg, row, word, o);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = ok ? bf2_poison(o[j]) : 0u;
    };
    uint32_t q[C::QREG ? 2 * KS : 1];
    // The queries in registers: asked for before the rows, behind which they would
    // come, and used when the rows are there.
    auto q_ask = [&](const Seg &sg) {
        if (!C::QREG) return;
        uint32_t o[WPT][4];
#pragma unroll
        for (int w = 0; w < WPT; ++w) q_load(sg, g, WPT * t + w, o[w]);
#pragma unroll
        for (int x = 0; x < 4 * WPT; ++x) q[C::QREG ? x : 0] = o[x >> 2][x & 3];
    };
    auto q_use = [&](bool ok) {
#pragma unroll
        for (int x = 0; x < (C::QREG ? 2 * KS : 0); ++x) q[C::QREG ? x : 0] = ok ? bf2_poison(q[C::QREG ? x : 0]) : 0u;
    };
    auto q_info = [&](const Seg &sg, int to) {  // token and position of the rows
        if (tid >= R) return;
        const int r = sg.rt * R + tid, i = r / a.G;
        const bool ok = r < a.n * a.G && sg.key.live && i < sg.key.cnt;
        rowinfo[to][tid] = ok ? make_int2(i, kv4_pos(sg.key.P, a.mask ? a.depth + sg.b * a.depth_b : nullptr, i)) : make_int2(-1, 0);
    };
    q_ask(cur);
    int mine = my_tiles(cur);
    for (int y = 0; y < min(ST, mine); ++y) issue(cur, y, seq + y);

    q_info(cur, 0);
    __syncthreads();
    int info = 0;  // which of the two is this segment's
    bool first = true;
    while (true) {
        const Kv4Keys key = cur.key;
        const int b = cur.b, rt = cur.rt, h = cur.h, P = key.P, end = P + key.cnt;
        const int2 *rows = rowinfo[info];
        q_use(rows[g].x >= 0);
        if (!C::QREG) {
            for (int x = tid; x < NT * SPL * (KS / 2) * 32; x += FT) {  // one word: two steps of a lane
                const int l = x & 31, w = (x >> 5) % WPT, sp = (x >> 5) / WPT % SPL, nt = (x >> 5) / WPT / SPL;
                uint32_t o[4];
                q_words(cur, nt * 8 + (l >> 2), WPT * (l & 3) + w, sp, o);
                qs[((nt * SPL + sp) * KS + 2 * w) * 32 + l] = make_uint2(o[0], o[1]);
                qs[((nt * SPL + sp) * KS + 2 * w + 1) * 32 + l] = make_uint2(o[2], o[3]);
            }
        }
        if (!C::QREG) __syncthreads();
        int posmax = 0;
        if (a.window)
            for (int r = 0; r < R; ++r) posmax = max(posmax, rows[r].y);
        const int all_see = P + (a.mask ? 0 : key.i0 + 1);  // positions below it are new to no row

        float O[NT][JT][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
            for (int j = 0; j < JT; ++j) O[nt][j][0] = O[nt][j][1] = O[nt][j][2] = O[nt][j][3] = 0.0f;
        }
        for (int y = 0; y < mine; ++y, ++seq) {
            const int s = seq % ST;
            if (!bad && !mbar_wait(bar0 + 8 * s, (seq / ST) & 1)) {
                bad = true;  // no more copies; those under way are waited for before the end
                mbar_drain<ST>(bar0, seq);
            }
            const uint8_t *kt = ringp + s * C::STAGE, *vt = kt + FKT * RB;
            const int j0 = kv4_tile<FKT>(key, (cur.x0 + y) * FW + warp);
            float S[NT][2][4];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) S[nt][mt][0] = S[nt][mt][1] = S[nt][mt][2] = S[nt][mt][3] = 0.0f;
                uint32_t w[2][WPT], t2[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint8_t *row = kt + (mt * 16 + x * 8 + g) * RB;
                    if (WPT == 4) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(row + 16 * t);
                        w[x][0] = v.x, w[x][1] = v.y, w[x][WPT / 2] = v.z, w[x][WPT - 1] = v.w;
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2 *>(row + 8 * t);
                        w[x][0] = v.x, w[x][1] = v.y;
                    }
                    t2[x] = *reinterpret_cast<const uint32_t *>(row + D / 2 + 4 * t) & KV4_T_MASK;
                }
#pragma unroll
                for (int i = 0; i < WPT; ++i) {
                    uint32_t p[2][4];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const uint32_t tt = __byte_perm(t2[x], 0, i < WPT / 2 ? 0x1010 : 0x3232);
                        kv4_pairs(w[x][i], tt, kv4_offset(tt), p[x]);
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const uint32_t A[4] = {p[0][2 * u], p[1][2 * u], p[0][2 * u + 1], p[1][2 * u + 1]};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            if (C::QREG) {
                                mma16816(S[nt][mt], A, q[C::QREG ? 4 * i + 2 * u : 0], q[C::QREG ? 4 * i + 2 * u + 1 : 0]);
                            } else {
#pragma unroll
                                for (int sp = SPL - 1; sp >= 0; --sp) {
                                    const uint2 qq = qs[((nt * SPL + sp) * KS + 2 * i + u) * 32 + lane];
                                    mma16816(S[nt][mt], A, qq.x, qq.y);
                                }
                            }
                        }
                    }
                }
            }
            // scores to weights
            const bool masked = j0 + FKT > all_see || (a.window && j0 <= posmax - a.window && j0 + FKT > a.sinks);
            uint32_t pk[NT][2][SPL][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (masked) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int2 ri = rows[nt * 8 + 2 * t + c];
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                            for (int x = 0; x < 2; ++x)
                                if (ri.x < 0 || !kv4_sees(a, b, P, end, j0 + mt * 16 + x * 8 + g, ri.x, ri.y))
                                    S[nt][mt][2 * x + c] = -INFINITY;
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float mx = fmaxf(fmaxf(S[nt][0][c], S[nt][0][2 + c]), fmaxf(S[nt][1][c], S[nt][1][2 + c])) * a.scale;
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                    // (rescaled only when the maximum grew by more than 2^8: weights stay below
                    // that and lose nothing by it)
                    float mn = mx > m[nt][c] + F_LAZY || m[nt][c] == -INFINITY ? fmaxf(m[nt][c], mx) : m[nt][c];
                    if (__any_sync(0xffffffffu, mn > m[nt][c])) {
                        const float f = mn == -INFINITY ? 1.0f : ex2(m[nt][c] - mn);
                        m[nt][c] = mn;
                        l[nt][c] *= f;
#pragma unroll
                        for (int j = 0; j < JT; ++j) O[nt][j][c] *= f, O[nt][j][2 + c] *= f;
                    }
                    const float ref = mn == -INFINITY ? 0.0f : mn;
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const float p = ex2(fmaf(S[nt][mt][2 * x + c], a.scale, -ref));
                            S[nt][mt][2 * x + c] = p;
                            l[nt][c] += p;
                        }
                }
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float p0 = S[nt][mt][2 * x], p1 = S[nt][mt][2 * x + 1];
#pragma unroll
                        for (int sp = 0; sp < SPL; ++sp) {
                            const uint32_t w = bf2_pack(p0, p1);
                            pk[nt][mt][sp][x] = movmatrix(w);
                            p0 -= bf_lo(w), p1 -= bf_hi(w);
                        }
                    }
            }
            // values
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                uint32_t w[4][WPT / 2], t1[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint8_t *row = vt + (mt * 16 + 2 * t + (x & 1) + (x >> 1) * 8) * RB;
                    if (WPT == 4) {
                        const uint2 v = *reinterpret_cast<const uint2 *>(row + 8 * g);
                        w[x][0] = v.x, w[x][WPT / 2 - 1] = v.y;
                    } else {
                        w[x][0] = *reinterpret_cast<const uint32_t *>(row + 4 * g);
                    }
                    t1[x] = *reinterpret_cast<const unsigned short *>(row + D / 2 + 2 * g);
                }
                // pairs of neighbouring keys: lo[u] of keys 2t, 2t + 1, then of 2t + 8, 2t + 9
                uint32_t tt[2], off[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    tt[u] = __byte_perm(t1[2 * u], t1[2 * u + 1], 0x5410) & KV4_T_MASK;
                    off[u] = kv4_offset(tt[u]);
                }
                // even and odd channels of a word: pv[word][odd][u][j]
                uint32_t pv[WPT / 2][2][2][4];
#pragma unroll
                for (int i = 0; i < WPT / 2; ++i)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        kv4_pairs(__byte_perm(w[2 * u][i], w[2 * u + 1][i], 0x5410), tt[u], off[u], pv[i][0][u]);
                        kv4_pairs(__byte_perm(w[2 * u][i], w[2 * u + 1][i], 0x7632), tt[u], off[u], pv[i][1][u]);
                    }
                // D = 128: rows g are word 2g, rows g + 8 word 2g + 1; D = 64: channels j and j + 4 of word g
#pragma unroll
                for (int j = 0; j < JT; ++j) {
                    constexpr int I1 = WPT / 2 - 1;
                    const int ja = j, jb = WPT == 4 ? j : j + 4;
                    const uint32_t A[4] = {pv[0][ja & 1][0][ja >> 1], pv[I1][jb & 1][0][jb >> 1], pv[0][ja & 1][1][ja >> 1],
                                           pv[I1][jb & 1][1][jb >> 1]};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (F32) {  // the products of 16 keys are summed apart: the tensor cores' sums do not round to nearest
                            float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                            for (int sp = SPL - 1; sp >= 0; --sp) mma16816(c, A, pk[nt][mt][sp][0], pk[nt][mt][sp][1]);
#pragma unroll
                            for (int x = 0; x < 4; ++x) O[nt][j][x] += c[x];
                        } else {
                            mma16816(O[nt][j], A, pk[nt][mt][0][0], pk[nt][mt][0][1]);
                        }
                    }
                }
            }
            // The next copy into this place comes after these loads only if they are over:
            // a fence between the two kinds of access.
            async_fence();
            __syncwarp();
            if (y + ST < mine) issue(cur, y + ST, seq + ST);
        }
        // the next segment, whose first tiles are on their way while this one is merged
        const bool whole = CL <= 1 && cur.whole();
        const bool more = cur.next(a, R, RT);
        mine = more ? my_tiles(cur) : 0;
        if (more) {
            place_rows(cur);
            q_ask(cur);
        }
        for (int y = 0; y < min(ST, mine); ++y) issue(cur, y, seq + y);
        if (more) q_info(cur, info ^ 1);
        // merge the warps
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 4);
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 8);
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 16);
                if (g == 0) sm_m[warp][nt * 8 + 2 * t + c] = m[nt][c], sm_l[warp][nt * 8 + 2 * t + c] = l[nt][c];
            }
        if (bad && lane == 0) any_timeout = 1;
        __syncthreads();
        // (a cluster's parts stay in the rings, whose tiles are all used)
        float *slot = CL > 1 ? reinterpret_cast<float *>(smem) : ws.piece + (size_t)(2 * blockIdx.x + (first ? 0 : 1)) * R * (D + 2);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float M[2], L[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                M[c] = sm_m[0][nt * 8 + 2 * t + c];
                for (int w = 1; w < FW; ++w) M[c] = fmaxf(M[c], sm_m[w][nt * 8 + 2 * t + c]);
                const float ref = M[c] == -INFINITY ? 0.0f : M[c];
                L[c] = 0.0f;
                for (int w = 0; w < FW; ++w) L[c] += sm_l[w][nt * 8 + 2 * t + c] * ex2(sm_m[w][nt * 8 + 2 * t + c] - ref);
                const float f = ex2(m[nt][c] - ref);
#pragma unroll
                for (int j = 0; j < JT; ++j) {
                    merge[((warp * JT + j) * 4 + c) * 32 + lane] = O[nt][j][c] * f;
                    merge[((warp * JT + j) * 4 + 2 + c) * 32 + lane] = O[nt][j][2 + c] * f;
                }
            }
            __syncthreads();
            if (warp < JT) {  // warp j adds up the j-th tile of channels
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    float o = 0.0f;
#pragma unroll
                    for (int w = 0; w < FW; ++w) o += merge[((w * JT + warp) * 4 + x) * 32 + lane];
                    const int c = x & 1, row = nt * 8 + 2 * t + c, r = rt * R + row;
                    const int d = WPT == 4 ? 16 * g + (x >> 1) * 8 + warp : 8 * g + (x >> 1) * 4 + warp;
                    const int i = r / a.G;
                    if (!whole) {
                        slot[row * D + d] = o;
                    } else if (r < a.n * a.G) {
                        const float v = L[c] == 0.0f || rows[row].x < 0 ? 0.0f : o * KV4_STEP / L[c];
                        const size_t at_o = (((size_t)b * a.n + i) * a.Hq + h * a.G + r % a.G) * D + d;
                        if (F32)
                            reinterpret_cast<float *>(a.out)[at_o] = v;
                        else
                            reinterpret_cast<__nv_bfloat16 *>(a.out)[at_o] = __float2bfloat16_rn(v);
                    }
                }
            }
            if (warp == 0 && g == 0) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int row = nt * 8 + 2 * t + c, r = rt * R + row, i = r / a.G;
                    if (!whole) {
                        slot[R * D + row] = M[c];
                        slot[R * D + R + row] = L[c];
                    } else if (a.lse && r < a.n * a.G) {
                        a.lse[((size_t)b * a.n + i) * a.Hq + h * a.G + r % a.G] =
                            L[c] == 0.0f || rows[row].x < 0 ? -INFINITY : (M[c] + log2f(L[c])) * 0.6931471805599453f;
                    }
                }
            }
            __syncthreads();  // before the next rows' sums, the next segment's row infos and its maxima
        }
        first = false;
        info ^= 1;
        if (!more) break;
    }
    if (CL > 1) {  // the cluster's parts, in their order
        constexpr int D4 = D / 4;
        cluster_sync();
        const int e = rank * FT + tid, row = e / D4, d4 = e % D4;
        if (row < R) {
            const uint32_t box = smem_u32(smem);
            float4 v[FCL];
            float m[FCL], l[FCL], top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int c = 0; c < FCL; ++c) {
                m[c] = -INFINITY, l[c] = 0.0f;
                if (c >= CL) continue;
                const uint32_t at_c = cluster_map(box, c);
                m[c] = cluster_ld(at_c + 4 * (R * D + row)), l[c] = cluster_ld(at_c + 4 * (R * D + R + row));
                v[c] = cluster_ld4(at_c + 16 * (row * D4 + d4));
            }
#pragma unroll
            for (int c = 0; c < FCL; ++c) top = fmaxf(top, m[c]);
            const float ref = top == -INFINITY ? 0.0f : top;
            float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int c = 0; c < FCL; ++c) {
                if (c >= CL) continue;
                const float f = ex2(m[c] - ref);
                sum = fmaf(l[c], f, sum);
                o.x = fmaf(v[c].x, f, o.x), o.y = fmaf(v[c].y, f, o.y), o.z = fmaf(v[c].z, f, o.z), o.w = fmaf(v[c].w, f, o.w);
            }
            const int r = at.rt * R + row, i = r / a.G;
            if (r < a.n * a.G) {
                const bool none = sum == 0.0f || rowinfo[0][row].x < 0;
                const float k = none ? 0.0f : KV4_STEP / sum;
                const size_t orow = ((size_t)at.b * a.n + i) * a.Hq + at.h * a.G + r % a.G;
                if (none) o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (F32)
                    reinterpret_cast<float4 *>(a.out)[orow * D4 + d4] = make_float4(o.x * k, o.y * k, o.z * k, o.w * k);
                else
                    reinterpret_cast<uint2 *>(a.out)[orow * D4 + d4] = make_uint2(bf2_pack(o.x * k, o.y * k), bf2_pack(o.z * k, o.w * k));
                if (d4 == 0 && a.lse) a.lse[orow] = none ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
            }
        }
        cluster_sync();  // nobody leaves while its part is read
    }
    if (tid == 0 && any_timeout) {
        if (direct)
            atomicOr(a.status + at.b, ACES_ROW_TIMEOUT);  // seconds after it was written
        else
            ws.info[blockIdx.x].timeout = 1;
    }
}

// Adds the pieces of an item that several CTAs share, in their order: block
// group c (Y blocks) takes the item in which the range of CTA c starts, when c is
// the first to start inside it.  Block 0 writes the sequences' status.  The grid
// is launched while the attention runs and waits for its end.
// A warp takes four rows, eight lanes each, three pieces at a time with all their
// loads under way at once.  Many pieces of up to 16 rows (one long sequence): the
// block takes a row and its warps every eighth piece.  What bounds it is its start
// and two dependent loads: 10.5 us for the 23.5 MB of 152 items of 256 rows of 128
// (a warp a row, two at a time: 14.1), 7.6 for 300 of four rows, with cold caches.
constexpr int JN = 256, JW = JN / 32;
template <int D, bool F32>
__global__ void __launch_bounds__(JN) k_kv4_join(Kv4Att a, Kv4Ws ws, int C, int R, int Y) {
    constexpr int D4 = D / 4, PW = 32 / D4;  // float4 of a row; pieces a warp reads at a time
    __shared__ int late;
    __shared__ float4 part[JW][D4];
    __shared__ float part_m[JW], part_l[JW];
    const int tid = threadIdx.x, c = blockIdx.x / Y, y = blockIdx.x - c * Y, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    if (c == 0) {
        if (y != 0) return;
        if (tid == 0) late = 0;
        __syncthreads();
        for (int x = tid; x < C; x += JN)
            if (ws.info[x].timeout) late = 1;
        __syncthreads();
        for (int b = tid; b < a.B; b += JN)
            a.status[b] = (kv4_seq(a.prefix, a.count, b, a.n, a.S).ok ? 0 : ACES_ROW_RANGE) | (late ? ACES_ROW_TIMEOUT : 0);
        return;
    }
    const Kv4Info in = ws.info[c];
    // inside the item, and the first to start there
    if (in.cnt < 0 || in.off < in.inside || in.off - in.quantum >= in.inside) return;
    const int pieces = 1 + (in.all - in.off + in.quantum - 1) / in.quantum;
    const int stride = R * (D + 2), NR = min(R, a.n * a.G - in.rt * R);
    const float *first = ws.piece + (size_t)(2 * (c - 1) + (in.off >= in.quantum ? 0 : 1)) * stride;
    const float *rest = ws.piece + (size_t)(2 * (c - 1)) * stride;  // piece p > 0 at 2 p strides
    auto piece = [&](int p) { return p == 0 ? first : rest + (size_t)(2 * p) * stride; };
    // Pieces p0, p0 + step ... of a row: their sums to the maximum of them all, in
    // lanes 0 .. D4 - 1, and the sum of the weights.
    auto add = [&](int row, int p0, int step, float &M, float &L) {
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        M = -INFINITY, L = 0.0f;
        for (int base = p0; base < pieces; base += 32 * step) {
            const int mine = base + lane * step;
            float m = -INFINITY, l = 0.0f;
            if (mine < pieces) m = piece(mine)[R * D + row], l = piece(mine)[R * D + R + row];
            const int np = min(32, (pieces - base + step - 1) / step);
            const float top = fmaxf(M, warp_max(m)), ref = top == -INFINITY ? 0.0f : top;
            const float f = ex2(m - ref), old = ex2(M - ref);
            M = top;
            L = L * old + l * f;
            o.x *= old, o.y *= old, o.z *= old, o.w *= old;
#pragma unroll 8
            for (int q = 0; q < np; q += PW) {
                const int p = q + lane / D4;
                const float fp = __shfl_sync(0xffffffffu, f, p & 31);
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (p < np) v = *reinterpret_cast<const float4 *>(piece(base + p * step) + row * D + 4 * (lane % D4));
                if (p < np) o.x = fmaf(v.x, fp, o.x), o.y = fmaf(v.y, fp, o.y), o.z = fmaf(v.z, fp, o.z), o.w = fmaf(v.w, fp, o.w);
            }
        }
        for (int x = 16; x > 0; x >>= 1) L += __shfl_xor_sync(0xffffffffu, L, x);
        if (PW == 2) {
            o.x += __shfl_xor_sync(0xffffffffu, o.x, 16), o.y += __shfl_xor_sync(0xffffffffu, o.y, 16);
            o.z += __shfl_xor_sync(0xffffffffu, o.z, 16), o.w += __shfl_xor_sync(0xffffffffu, o.w, 16);
        }
        return o;
    };
    auto put = [&](int row, int d4, float4 o, float M, float L) {
        const int r = in.rt * R + row, i = r / a.G;
        const bool none = L == 0.0f || i >= in.cnt;
        const float k = none ? 0.0f : KV4_STEP / L;
        if (none) o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const size_t orow = ((size_t)in.b * a.n + i) * a.Hq + in.h * a.G + (r - i * a.G);
        if (F32)
            reinterpret_cast<float4 *>(a.out)[orow * D4 + d4] = make_float4(o.x * k, o.y * k, o.z * k, o.w * k);
        else
            reinterpret_cast<uint2 *>(a.out)[orow * D4 + d4] = make_uint2(bf2_pack(o.x * k, o.y * k), bf2_pack(o.z * k, o.w * k));
        if (d4 == 0 && a.lse) a.lse[orow] = none ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
    };
    if (pieces <= 3 || NR > 16) {
        constexpr int LN = 8, RW = 32 / LN, V = D4 / LN;  // lanes of a row, rows of a warp
        const int d4 = lane % LN;
        for (int row0 = (y * JW + warp) * RW; row0 < NR; row0 += Y * JW * RW) {
            const int row = row0 + lane / LN, rd = min(row, NR - 1);
            float top = -INFINITY, sum = 0.0f;
            float4 o[V];
#pragma unroll
            for (int x = 0; x < V; ++x) o[x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int p0 = 0; p0 < pieces; p0 += 3) {
                float4 v[3][V];
                float m[3], l[3];
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    const float *pc = piece(min(p0 + p, pieces - 1));
                    m[p] = pc[R * D + rd], l[p] = pc[R * D + R + rd];
#pragma unroll
                    for (int x = 0; x < V; ++x) v[p][x] = *reinterpret_cast<const float4 *>(pc + rd * D + 4 * (d4 + x * LN));
                }
                const float was = top;
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    if (p0 + p < pieces) top = fmaxf(top, m[p]);
                const float ref = top == -INFINITY ? 0.0f : top, old = ex2(was - ref);
                sum *= old;
#pragma unroll
                for (int x = 0; x < V; ++x) o[x].x *= old, o[x].y *= old, o[x].z *= old, o[x].w *= old;
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    if (p0 + p >= pieces) break;
                    const float f = ex2(m[p] - ref);
                    sum = fmaf(l[p], f, sum);
#pragma unroll
                    for (int x = 0; x < V; ++x)
                        o[x].x = fmaf(v[p][x].x, f, o[x].x), o[x].y = fmaf(v[p][x].y, f, o[x].y), o[x].z = fmaf(v[p][x].z, f, o[x].z),
                        o[x].w = fmaf(v[p][x].w, f, o[x].w);
                }
            }
            if (row < NR)
#pragma unroll
                for (int x = 0; x < V; ++x) put(row, d4 + x * LN, o[x], top, sum);
        }
    } else {
        for (int row = y; row < NR; row += Y) {
            float M, L;
            const float4 o = add(row, warp, JW, M, L);
            if (lane < D4) part[warp][lane] = o;
            if (lane == 0) part_m[warp] = M, part_l[warp] = L;
            __syncthreads();
            if (tid < D4) {
                float top = part_m[0], sum = 0.0f;
                for (int w = 1; w < JW; ++w) top = fmaxf(top, part_m[w]);
                const float ref = top == -INFINITY ? 0.0f : top;
                float4 all = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                for (int w = 0; w < JW; ++w) {
                    const float f = ex2(part_m[w] - ref);
                    const float4 v = part[w][tid];
                    sum = fmaf(part_l[w], f, sum);
                    all.x = fmaf(v.x, f, all.x), all.y = fmaf(v.y, f, all.y), all.z = fmaf(v.z, f, all.z), all.w = fmaf(v.w, f, all.w);
                }
                put(row, tid, all, top, sum);
            }
            __syncthreads();
        }
    }
}

cudaError_t launch_kv4_join(const Kv4Att &a, const Kv4Ws &ws, int C, int R, cudaStream_t s) {
    const int rows = a.n * a.G < R ? a.n * a.G : R;
    const int Y = rows <= 16 ? rows : (rows + 31) / 32;  // blocks of an item
    const auto fn = a.D == 64 ? (a.f32 ? k_kv4_join<64, true> : k_kv4_join<64, false>) : (a.f32 ? k_kv4_join<128, true> : k_kv4_join<128, false>);
    return launch_after(fn, C * Y, JN, 1, s, a, ws, C, R, Y);
}

// CTAs of a cluster that has an item to itself, or 0: shares and a join.  An item's
// units are counted by the cache's length or the window's (the sequences' lengths lie
// on the device): in a cache that is longer than it needs to be, shares come sooner.
//   Two to eight CTAs, while there is an SM for each (beyond, two on an SM take longer:
// four sequences of 4000 positions, eight key heads, by fours 18.5 us, by eights 20.5)
// and none has more than KV4_DIRECT units.  Against shares (us, eight key heads of 128):
// one sequence of 1000 positions 12.4 / 14.3, of 4000 14.8 / 16.4, of 8000 16.9 / 20.5,
// of 16000 22.6 / 24.6 (by eights); four of 8000 22.7 / 27.6 (by fours).
//   One CTA, up to KV4_DIRECT units, for any number of items of bfloat16.  Against
// shares (key heads of 128, sequences as long as the cache, and in brackets of all
// lengths up to it): four rows, 152 items of eight units 20.6 / 28.6 (20.6 / 24.0), 320
// 41.0 / 40.9 (29.5 / 30.9), 640 63.5 / 64.7 (47.9 / 48.0), 1216 98.8 / 100.5 (77.9 /
// 76.0), 320 of two units 20.6 / 24.5; 16 rows, one CTA an SM, 160 of eight 49.1 / 40.9
// (28.7 / 34.8), 320 73.5 / 64.0 (47.3 / 53.0).  Float32's products are three times as
// many, and a last wave that is nearly empty costs more than a join: beyond the SMs'
// number up to FEW_ONE units.  160 of eight 46.0 / 34.9 (26.1 / 29.7), 320 69.7 / 59.4
// (43.0 / 43.1), 512 92.9 / 85.8 (65.6 / 61.5); of four 160 30.7 / 26.9 (19.7 / 23.0),
// 320 45.1 / 40.8 (31.9 / 34.9); of two 22.1 / 22.6 (18.5 / 22.3), 31.3 / 31.3 (26.8 /
// 30.8).
constexpr int FEW_ONE = 4;
static int few_cluster(long long items, int most, bool f32, int nsm) {
    int cl = 1;
    while (cl < FCL && cl < most && items * cl * 2 <= nsm) cl *= 2;
    if (items >= (1ll << 30) || (most + cl - 1) / cl > KV4_DIRECT) return 0;
    return f32 && items > nsm && most > FEW_ONE ? 0 : cl;
}

template <int D, bool F32, int NT>
static cudaError_t run_few(const Kv4Att &a, void *workspace, int nsm, cudaStream_t s) {
    using C = Few<D, F32, NT>;
    const int RT = (int)(((long long)a.n * a.G + C::R - 1) / C::R);
    const long long items = (long long)a.B * RT * a.H;
    const int most = kv4_most_units(a, FW * FKT), CL = few_cluster(items, most, F32, nsm);
    const bool direct = CL > 0;
    const int grid = direct ? (int)items * CL : nsm * C::MINB;
    const Kv4Ws ws = kv4_ws_carve(workspace, nsm * C::MINB);
    static std::atomic<unsigned long long> allowed{0};
    cudaError_t e = allow_smem(k_kv4_few<D, F32, NT>, C::SMEM, allowed);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid), cfg.blockDim = dim3(FT), cfg.dynamicSmemBytes = C::SMEM, cfg.stream = s;
    cudaLaunchAttribute shape;
    shape.id = cudaLaunchAttributeClusterDimension;
    shape.val.clusterDim.x = direct ? CL : 1, shape.val.clusterDim.y = shape.val.clusterDim.z = 1;
    cfg.attrs = &shape, cfg.numAttrs = CL > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, k_kv4_few<D, F32, NT>, a, ws, RT, CL);
    return e != cudaSuccess || direct ? e : launch_kv4_join(a, ws, grid, C::R, s);
}

// Rows of a tile: 8 when a head's rows fit (or float32 has few), else 16.
static int few_tiles(int n, int G) { return (long long)n * G <= 8 ? 1 : 2; }

size_t kv4_few_ws(int n, int G, int D, int nsm) { return kv4_ws_bytes(2 * nsm, 8 * few_tiles(n, G), D); }

cudaError_t launch_kv4_few(const Kv4Att &a, void *workspace, int nsm, cudaStream_t s) {
    const bool one = few_tiles(a.n, a.G) == 1;
    if (a.D == 64)
        return a.f32 ? (one ? run_few<64, true, 1>(a, workspace, nsm, s) : run_few<64, true, 2>(a, workspace, nsm, s))
                     : (one ? run_few<64, false, 1>(a, workspace, nsm, s) : run_few<64, false, 2>(a, workspace, nsm, s));
    return a.f32 ? (one ? run_few<128, true, 1>(a, workspace, nsm, s) : run_few<128, true, 2>(a, workspace, nsm, s))
                 : (one ? run_few<128, false, 1>(a, workspace, nsm, s) : run_few<128, false, 2>(a, workspace, nsm, s));
}

#ifdef ACES_CHECKED
cudaError_t check_take_kv4_few(unsigned long long out[3]) { return check_take(out); }
#endif

}  // namespace aces
