// How the attention kernels share their work out (both read kv4.cuh's arguments).
//
// An item is one tile of R query rows (row r = token r / G, head r % G of the
// group) of one sequence and key head; its keys are cut into tiles, and some
// tiles are a unit.  The sequences' lengths lie on the device, so every CTA
// counts the units of all items itself (one thread an entry (b, row tile), all
// of whose heads have the same) and takes the units [c Q, (c + 1) Q), Q the
// whole number that spreads them over the grid: CTAs are equally long whatever
// the lengths.  Units are counted by their time (Cost::weight), and what an item
// costs beside its keys (its queries, its merge, its way out) counts as Cost::FIX
// before its first: without, a CTA that got the short sequences of a ragged
// batch took twice the others' time.  An item inside
// one CTA's range is written out by it; the pieces of one that several share go
// to the workspace as sums not yet divided, with their reference maximum, and
// k_kv4_join adds them in the CTAs' order.
// Where no item can have more than KV4_DIRECT units for each CTA of a cluster, or one
// CTA (the cache is short, or the window), it takes the item and adds its parts up in
// shared memory: nothing to join (few rows only: few_cluster() and its figures).
#pragma once
#include <atomic>

#include "kv4.cuh"

namespace aces {

constexpr int KV4_DIRECT = 8;

struct Kv4Info {  // of the item in which a CTA's range starts
    int b, rt, h;
    int off, all;  // where in the item, of what in all, in the measure of Cost
    int inside;    // the least `off` that lies beyond its first unit
    int quantum;
    int cnt;      // the sequence's tokens (0: none in the cache); -1: the CTA has nothing to do
    int timeout;
    int pad[3];
};
static_assert(sizeof(Kv4Info) == 48, "Kv4Info layout");

// Workspace: Kv4Info[C], then 2 C pieces of R * (D + 2) floats (a CTA's first
// piece and its last).
struct Kv4Ws {
    Kv4Info *info;
    float *piece;
    float *total;  // k_kv4_many's own
};
inline size_t kv4_ws_bytes(int C, int R, int D) { return sizeof(Kv4Info) * (size_t)C + (size_t)2 * C * R * (D + 2) * 4; }
inline Kv4Ws kv4_ws_carve(void *p, int C) {
    Kv4Ws w;
    w.info = reinterpret_cast<Kv4Info *>(p);
    w.piece = reinterpret_cast<float *>(w.info + C);
    w.total = nullptr;
    return w;
}

// Keys of one row tile of one sequence: those below s_hi (the first tokens
// that stay visible) and [lo, hi), in tiles of KT.
struct Kv4Keys {
    int P, cnt, i0, i1;    // tokens [i0, i1]
    int lo, hi, s_hi;
    int st, mt0, tiles, units;
    int rows;              // of the tile
    bool live;
};

template <int KT, int TPU>
__device__ __forceinline__ Kv4Keys kv4_keys(const Kv4Att &a, int R, const Kv4Seq &sq, int rt) {
    Kv4Keys k;
    k.P = sq.P, k.cnt = sq.cnt;
    const int r0 = rt * R, r1 = min(r0 + R, a.n * a.G);  // at most 2^30 rows
    k.rows = r1 - r0;
    k.i0 = r0 / a.G;
    k.i1 = min((r1 - 1) / a.G, sq.cnt - 1);
    k.live = sq.ok && k.i0 < sq.cnt;
    k.lo = k.hi = k.s_hi = k.st = k.mt0 = k.tiles = 0;
    if (k.live) {
        k.hi = k.P + (a.mask ? k.cnt : k.i1 + 1);
        k.lo = a.window ? max(0, k.P + (a.mask ? 0 : k.i0) - a.window + 1) : 0;
        k.s_hi = min(a.sinks, k.lo);
        k.st = (k.s_hi + KT - 1) / KT;
        k.mt0 = max(k.lo / KT, k.st);
        k.tiles = k.st + max(0, (k.hi + KT - 1) / KT - k.mt0);
    }
    k.units = max(1, (k.tiles + TPU - 1) / TPU);
    return k;
}
template <int KT, int TPU>
__device__ __forceinline__ Kv4Keys kv4_keys(const Kv4Att &a, int R, int b, int rt) {
    return kv4_keys<KT, TPU>(a, R, kv4_seq(a.prefix, a.count, b, a.n, a.S), rt);
}
// first key of the x-th tile
template <int KT>
__device__ __forceinline__ int kv4_tile(const Kv4Keys &k, int x) {
    return (x < k.st ? x : k.mt0 + x - k.st) * KT;
}

// Whether new or old position j is seen by token i at position pos.
__device__ __forceinline__ bool kv4_sees(const Kv4Att &a, int b, int P, int end, int j, int i, int pos) {
    if (j >= end) return false;
    int kp = j;
    if (j >= P) {
        const int t = j - P;
        if (a.mask) {
            if (!((__ldg(a.mask + b * a.mask_b + (size_t)i * a.words + (t >> 5)) >> (t & 31)) & 1u)) return false;
            kp = kv4_pos(P, a.depth + b * a.depth_b, t);
        } else if (t > i) {
            return false;
        }
    }
    return !a.window || kp > pos - a.window || kp < a.sinks;
}

// A CTA's range and the item it starts in, by all NTH threads.  off and left are
// in the measure of Cost.
struct Kv4Start {
    unsigned long long left;
    int quantum, b, rt, h, off, cnt;
    Kv4Keys key;
};
template <int KT, int TPU, class Cost, int NTH>
__device__ __forceinline__ Kv4Start kv4_start(const Kv4Att &a, int R, int RT) {
    __shared__ unsigned long long red[NTH / 32];
    __shared__ Kv4Start found;
    const int E = a.B * RT, per = (E + NTH - 1) / NTH;
    const int e0 = min(E, (int)threadIdx.x * per), e1 = min(E, e0 + per);
    unsigned long long sum = 0, total;
    Kv4Keys k;
    for (int e = e0; e < e1; ++e) {
        k = kv4_keys<KT, TPU>(a, R, e / RT, e % RT);
        sum += (unsigned long long)Cost::all(k) * a.H;
    }
    unsigned long long at = block_exscan_n<NTH>(sum, red, &total);
    // (at least a unit's weight: no CTA between two others is left without one)
    const unsigned long long Q = max((total + gridDim.x - 1) / gridDim.x, (unsigned long long)Cost::MOST), w0 = Q * blockIdx.x;
    if (w0 >= at && w0 < at + sum) {
        for (int e = e0; e < e1; ++e) {
            if (per > 1) k = kv4_keys<KT, TPU>(a, R, e / RT, e % RT);
            const unsigned u = Cost::all(k);
            if (w0 < at + (unsigned long long)u * a.H) {
                const unsigned x = (unsigned)(w0 - at);
                found.b = e / RT, found.rt = e % RT, found.h = (int)(x / u), found.off = (int)(x % u);
                found.cnt = kv4_seq(a.prefix, a.count, found.b, a.n, a.S).ok ? k.cnt : 0;
                found.key = k;
                break;
            }
            at += (unsigned long long)u * a.H;
        }
    }
    __syncthreads();
    Kv4Start s = found;
    s.left = w0 < total ? min(Q, total - w0) : 0;
    s.quantum = (int)Q;
    return s;
}

// Without shares: a cluster of CL CTAs has the whole item.
template <int KT, int TPU, class Cost>
__device__ __forceinline__ Kv4Start kv4_whole(const Kv4Att &a, int R, int RT, int CL) {
    Kv4Start s;
    const int x = blockIdx.x / CL, e = x / a.H;
    s.h = x - e * a.H, s.b = e / RT, s.rt = e - s.b * RT;
    s.off = 0;
    s.key = kv4_keys<KT, TPU>(a, R, s.b, s.rt);
    s.left = s.quantum = Cost::all(s.key);
    s.cnt = s.key.cnt;
    if (threadIdx.x == 0 && s.h == 0 && s.rt == 0 && x * CL == blockIdx.x)
        a.status[s.b] = kv4_seq(a.prefix, a.count, s.b, a.n, a.S).ok ? 0 : ACES_ROW_RANGE;
    return s;
}
// the most units an item can have, by the cache's and the window's lengths
inline int kv4_most_units(const Kv4Att &a, int keys) {
    long long most = a.S;
    if (a.window) most = most < (long long)a.window + a.sinks + a.n + 2 * keys ? most : (long long)a.window + a.sinks + a.n + 2 * keys;
    return (int)((most + keys - 1) / keys);
}

// writes the info of the CTA's start (one thread)
template <class Cost>
__device__ __forceinline__ void kv4_put_info(const Kv4Ws &ws, const Kv4Start &at) {
    Kv4Info in;
    in.b = at.b, in.rt = at.rt, in.h = at.h, in.off = at.off, in.all = Cost::all(at.key), in.quantum = at.quantum;
    in.inside = Cost::FIX + Cost::weight(at.key);
    in.cnt = at.left > 0 ? at.cnt : -1;
    in.timeout = 0;
    ws.info[blockIdx.x] = in;
}

// A CTA's segments, one after another: units [x0, x1) of an item.
template <int KT, int TPU, class Cost>
struct Kv4Seg {
    unsigned long long left;  // after this segment, in the measure of Cost
    int b, rt, h, x0, x1;
    int next_P, next_cnt;     // of the next sequence, loaded long before they are wanted
    Kv4Keys key;
    __device__ __forceinline__ void ask(const Kv4Att &a) {
        const int nb = min(b + 1, a.B - 1);
        next_P = a.prefix[nb];
        next_cnt = a.count ? a.count[nb] : a.n;
    }
    __device__ __forceinline__ bool start(const Kv4Att &a, int R, int RT, const Kv4Start &at) {
        if (at.left == 0) return false;
        b = at.b, rt = at.rt, h = at.h, left = at.left, key = at.key;
        ask(a);
        return take(at.off);
    }
    __device__ __forceinline__ bool next(const Kv4Att &a, int R, int RT) {
        if (left == 0) return false;
        if (++h == a.H) {
            h = 0;
            Kv4Seq sq{key.P, key.cnt, true};
            if (++rt == RT) {
                rt = 0, ++b;
                sq.P = next_P, sq.cnt = next_cnt;
                ask(a);
            }
            sq.ok = sq.P >= 0 && sq.cnt >= 0 && sq.cnt <= a.n && (long long)sq.P + sq.cnt <= a.S;
            key = kv4_keys<KT, TPU>(a, R, sq, rt);
        }
        return take(0);
    }
    // From `off` of the item on, or as far as the range goes: a unit is the CTA's in
    // whose range the end of its weight lies.  False when the range ends before the
    // item's first unit does.
    __device__ __forceinline__ bool take(int off) {
        const int to = (int)min((unsigned long long)Cost::all(key), off + left), wt = Cost::weight(key);
        left -= to - off;
        x0 = max(off - Cost::FIX, 0) / wt, x1 = max(to - Cost::FIX, 0) / wt;
        return x1 > x0;
    }
    // first row of the item's key head in a plane
    __device__ __forceinline__ size_t row0(const Kv4Att &a) const { return (size_t)((size_t)b * a.H + h) * a.S; }
    __device__ __forceinline__ bool whole() const { return x0 == 0 && x1 == key.units; }
};

// Lets a kernel have that much shared memory, once on each of 64 devices.
template <typename F>
inline cudaError_t allow_smem(F *fn, int bytes, std::atomic<unsigned long long> &allowed) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev < 64 && (allowed.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) allowed.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

cudaError_t launch_kv4_join(const Kv4Att &a, const Kv4Ws &ws, int C, int R, cudaStream_t s);
size_t kv4_few_ws(int n, int G, int D, int nsm);
cudaError_t launch_kv4_few(const Kv4Att &a, void *workspace, int nsm, cudaStream_t s);
size_t kv4_many_ws(int n, int G, int D, int nsm);
cudaError_t launch_kv4_many(const Kv4Att &a, void *workspace, int nsm, cudaStream_t s);

// ---------------------------------------------------------------------------
// mbarriers and bulk copies
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok;
}
// Waits for a phase; gives up after two seconds (nothing it waits for takes a
// thousandth of that), so a mistake ends as a status and not as a hang.
constexpr unsigned long long KV4_WAIT_NS = 2000000000ull;
static __device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity) {
    const unsigned long long t0 = globaltimer_ns();
    while (!mbar_try(bar, parity))
        if (globaltimer_ns() - t0 > KV4_WAIT_NS) return false;
    return true;
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < 16; ++i)
        if (mbar_try(bar, parity)) return true;
    return mbar_wait_slow(bar, parity);
}
// global -> shared, 16-byte aligned, a multiple of 16 bytes
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

// this thread's plain shared-memory accesses before later copies and products
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---------------------------------------------------------------------------
// codes -> bfloat16 pairs
__device__ __forceinline__ uint32_t bf2_fma(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// -24 t of two t's (exact: two and five significant bits)
__device__ __forceinline__ uint32_t kv4_offset(uint32_t t2) { return bf2_fma(t2, 0xC1C0C1C0u, 0x80008000u); }
// a & 0x00780078 | 0x41804180 as one instruction (written in C it becomes two: an
// instruction has room for one of the constants)
__device__ __forceinline__ uint32_t kv4_sixteen(uint32_t a) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(a), "r"(0x00780078u), "r"(0x41804180u));
    return d;
}
// Four pairs of values from a word whose halves hold four codes each, pair j
// the codes at bits 4 j: a code at bits 3..6 of 16.0 makes 16 + c, and (16 + c)
// t - 24 t = (c - 8) t is exact.
__device__ __forceinline__ void kv4_pairs(uint32_t w, uint32_t t2, uint32_t off, uint32_t (&p)[4]) {
    p[0] = bf2_fma(kv4_sixteen(w << 3), t2, off);
    p[1] = bf2_fma(kv4_sixteen(w >> 1), t2, off);
    p[2] = bf2_fma(kv4_sixteen(w >> 5), t2, off);
    p[3] = bf2_fma(kv4_sixteen(w >> 9), t2, off);
}
// bfloat16 pair with infinities made NaN, so a query that is not finite spoils
// its row whatever the keys' signs
__device__ __forceinline__ uint32_t bf2_poison(uint32_t x) {
    if ((x & 0x7F80u) == 0x7F80u) x |= 0x40u;
    if ((x & 0x7F800000u) == 0x7F800000u) x |= 0x400000u;
    return x;
}
// low half from a, high half from b, rounded to nearest even
__device__ __forceinline__ uint32_t bf2_pack(float a, float b) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    return d;
}
__device__ __forceinline__ float bf_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf_hi(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }

}  // namespace aces
