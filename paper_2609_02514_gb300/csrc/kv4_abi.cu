// C entry points of the 4-bit KV cache: argument checks and launches.
#include <climits>

#include "kv4_plan.cuh"
#include "turn.cuh"

using namespace aces;

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// Checks of the cache, and the layer's two planes.
aces_status check_cache(const void *cache, int planes, int layer, int B, int H, int S, int D, uint8_t **k, uint8_t **v) {
    if (!cache || !aligned16(cache)) return ACES_ERR_INVALID_ARG;
    if (B < 1 || H < 1 || S < 1 || D < 1 || planes < 2 || layer < 0 || layer > planes / 2 - 1) return ACES_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return ACES_ERR_UNSUPPORTED;
    if ((long long)B * H > INT_MAX / 2 || S > INT_MAX / 4) return ACES_ERR_INVALID_ARG;
    const size_t plane = (size_t)B * H * S * kv4_row_bytes(D);
    uint8_t *base = reinterpret_cast<uint8_t *>(const_cast<void *>(cache));
    *k = base + 2 * (size_t)layer * plane;
    *v = *k + plane;
    return ACES_OK;
}

// every group of the strided numbers [B, n, H, D] starts on 16 bytes
bool on_grid(const void *p, const int64_t *stride, size_t es) {
    if (!aligned16(p)) return false;
    for (int i = 0; i < 3; ++i)
        if ((stride[i] * (int64_t)es) % 16 != 0) return false;
    return true;
}

aces_status check_rows(const void *k, const void *v, aces_dtype dt, const int32_t *start, int B, int n, int H) {
    if (dt != ACES_F32 && dt != ACES_BF16) return ACES_ERR_UNSUPPORTED;
    if (!k || !v || !start || n < 1 || n > INT_MAX / 4) return ACES_ERR_INVALID_ARG;
    if ((long long)B * n > INT_MAX / 2 || (long long)n * H > INT_MAX / 64) return ACES_ERR_INVALID_ARG;
    const size_t es = dt == ACES_F32 ? 4 : 2;
    if ((uintptr_t)k % es || (uintptr_t)v % es) return ACES_ERR_INVALID_ARG;
    return ACES_OK;
}

// Which kernel: bfloat16 queries of more than 16 rows a key head go to the
// tcgen05 kernel, the others (and up to 32 rows of a few key heads, where latency
// counts) to the one that keeps its few rows in registers.  Measured (us, D = 128,
// eight key heads, few rows / tcgen05): 16 rows, 16 sequences of 16000 117 / 174,
// 64 of 4000 133 / 193; 32 rows, the same 211 / 177 and 244 / 197, and one
// sequence of 16000 33 / 37; 20 rows, one of 4000 20 / 27.
bool many_rows(int f32, int B, int H, int n, int G) {
    const long long rows = (long long)n * G;
    return !f32 && rows > ((long long)B * H <= 32 ? 32 : 16);
}

// Checks of an attention call beside its cache, and what they make of the kernels' arguments.
aces_status check_attention(const void *q, aces_dtype dt, const int64_t *q_strides, int B, int n, int Hq, int H, int D,
                            const int32_t *prefix_len, const uint32_t *mask, int64_t mask_stride, const int32_t *depth,
                            int64_t depth_stride, float scale, int window, int sinks, void *out, int32_t *seq_status, void *workspace,
                            Kv4Att *a) {
    if (dt != ACES_F32 && dt != ACES_BF16) return ACES_ERR_UNSUPPORTED;
    if (!q || !q_strides || !prefix_len || !out || !seq_status || !workspace) return ACES_ERR_INVALID_ARG;
    const size_t es = dt == ACES_F32 ? 4 : 2;
    if ((uintptr_t)q % es || !aligned16(out) || !aligned16(workspace)) return ACES_ERR_INVALID_ARG;
    if (n < 1 || Hq < H || Hq % H != 0) return ACES_ERR_INVALID_ARG;
    if ((mask == nullptr) != (depth == nullptr)) return ACES_ERR_INVALID_ARG;
    const int words = (n + 31) / 32;
    if (mask && ((mask_stride != 0 && mask_stride < (int64_t)n * words) || (depth_stride != 0 && depth_stride < n)))
        return ACES_ERR_INVALID_ARG;
    if (!(scale > 0.0f && scale <= 0x1p110f)) return ACES_ERR_INVALID_ARG;  // a.scale below is finite
    if (window < 0 || sinks < 0) return ACES_ERR_INVALID_ARG;
    *a = {};
    a->q = q;
    a->qb = q_strides[0], a->qi = q_strides[1], a->qh = q_strides[2];
    a->f32 = dt == ACES_F32;
    a->out = out, a->status = seq_status;
    a->prefix = prefix_len;
    a->mask = mask, a->mask_b = mask_stride, a->depth = depth, a->depth_b = depth_stride;
    a->B = B, a->n = n, a->Hq = Hq, a->H = H, a->G = Hq / H, a->D = D, a->words = words;
    a->window = window;
    a->sinks = window > 0 ? sinks : 0;
    a->scale = (float)((double)scale * 1.4426950408889634 * (double)KV4_STEP);
    return ACES_OK;
}

// Checks of what a rotation is, and its part of the kernel's arguments.
aces_status check_turn(const aces_turn *t, int D, int B, int n, int Hq, int H, const void *q, const void *k, aces_dtype dt, Turn *a) {
    if (D != 64 && D != 128) return D < 1 ? ACES_ERR_INVALID_ARG : ACES_ERR_UNSUPPORTED;
    if (dt != ACES_F32 && dt != ACES_BF16) return ACES_ERR_UNSUPPORTED;
    if (!t || !q || !k || !t->inv_freq || B < 1 || n < 1 || Hq < 1 || H < 1) return ACES_ERR_INVALID_ARG;
    if (n > INT_MAX / 4 || (long long)B * n > INT_MAX / 2 || Hq > INT_MAX / 64 || H > INT_MAX / 64) return ACES_ERR_INVALID_ARG;
    if (t->rot_dim < 1 || t->rot_dim > D) return ACES_ERR_INVALID_ARG;
    if (t->rot_dim % (D / 4) != 0) return ACES_ERR_UNSUPPORTED;
    if (t->positions && (t->n_axes < 1 || t->n_axes > ACES_MAX_AXES || (t->n_axes > 1 && !t->axes))) return ACES_ERR_INVALID_ARG;
    if (t->depth && t->depth_stride != 0 && t->depth_stride < n) return ACES_ERR_INVALID_ARG;
    if (!(t->scale >= 0x1p-20 && t->scale <= 0x1p20)) return ACES_ERR_INVALID_ARG;
    if (t->norm ? !(t->eps >= 1e-30 && t->eps <= 1.0) : (t->q_weight || t->k_weight)) return ACES_ERR_INVALID_ARG;
    const size_t es = dt == ACES_F32 ? 4 : 2;
    if ((uintptr_t)q % es || (uintptr_t)k % es) return ACES_ERR_INVALID_ARG;
    const void *w[2] = {t->q_weight, t->k_weight};
    const aces_dtype wt[2] = {t->q_weight_dt, t->k_weight_dt};
    const int64_t ws[2] = {t->q_weight_stride, t->k_weight_stride};
    for (int i = 0; i < 2; ++i) {
        TurnWeight &o = i ? a->kw : a->qw;
        o = {w[i], ws[i], wt[i] == ACES_F32, aligned16(w[i]) && ws[i] * (wt[i] == ACES_F32 ? 4 : 2) % 16 == 0};
        if (!w[i]) {
            o.h = 0;
            continue;
        }
        if (wt[i] != ACES_F32 && wt[i] != ACES_BF16) return ACES_ERR_UNSUPPORTED;
        if ((uintptr_t)w[i] % (o.f32 ? 4 : 2) || (ws[i] != 0 && ws[i] < D)) return ACES_ERR_INVALID_ARG;
    }
    a->freq = t->inv_freq, a->axes = t->axes, a->positions = t->positions;
    a->start = t->start, a->base = t->base, a->depth = t->depth, a->depth_b = t->depth_stride;
    a->R = t->rot_dim, a->n_axes = t->positions ? t->n_axes : 1, a->norm = t->norm;
    a->eps = t->eps, a->scale = t->scale;
    a->eps32 = (float)t->eps, a->eps_low = (float)(t->eps - a->eps32);
    a->scale32 = (float)t->scale, a->scale_low = (float)(t->scale - a->scale32);
    a->B = B, a->n = n, a->Hq = Hq, a->H = H;
    return ACES_OK;
}
// whether no two numbers of strided outputs [B, n, heads, D] share a place
bool apart(const int64_t *stride, int B, int n, int H, int D) {
    int64_t st[3] = {stride[0], stride[1], stride[2]}, size[3] = {B, n, H};
    int64_t least = D;
    for (int left = 3; left > 0; --left) {  // the smallest stride of what is left
        int at = -1;
        for (int i = 0; i < 3; ++i)
            if (size[i] > 0 && (at < 0 || st[i] < st[at])) at = i;
        if (size[at] > 1) {
            if (st[at] < least || st[at] > INT64_MAX / 4 / size[at]) return false;
            least = st[at] * size[at];
        }
        size[at] = 0;
    }
    return true;
}
TurnHeads heads(const void *p, const int64_t *s) { return {const_cast<void *>(p), s[0], s[1], s[2]}; }

// Whether a prefix's rows are worth a pass of their own: it saves every sequence's work
// on them but one's, and costs the parts' way through memory, more launches and a second
// set of items.  In microseconds, of the prefix's capacity or the window:
//   few rows: 256 keys of an item take a CTA 1.75, two CTAs an SM (float32 three times);
//   many: 128 keys of 256 rows 2.1 of an SM, of up to 128 rows two thirds of it.
// Measured (us, one pass / two; 32 heads over 8 of 128, 50 to 500 own positions; saved by
// the estimate in brackets): one token of 4 sequences behind 2000 positions 15 / 26 (1), of
// 16 29 / 31 (5), of 8 behind 8000 34 / 32 (9), of 32 behind 2000 40 / 36 (10), of 4 behind
// 32000 49 / 37 (17), of 16 behind 8000 54 / 36 (18); 20 tokens of 8 behind 8000 79 / 89
// (18), of 4 behind 32000 121 / 129 (28), of 16 behind 8000 131 / 119 (39); 80 tokens of 8
// behind 8000 191 / 189 (23), of 32 behind 2000 239 / 262 (23), of 16 behind 8000 347 / 326 (46).  Float32, 12 heads
// over 4 of 64: one token of 32 behind 2000 26 / 27 (14), of 8 behind 16000 33 / 31 (26).
// (The parts' way through memory, 1040 bytes a row of 128, is in the constants, though it grows with
// the rows: the two cases at 23 differ by it.)  A prefix that leaves its cache nearly empty
// pays for two passes all the same, 100 positions in a room of 16000 to 60000: one token of 16 sequences 12 / 22,
// of 64 26 / 39; float32 11 / 22, 43 / 57; 80 tokens of 16 58 / 86, of 64 173 / 226.
constexpr double FEW_EXTRA = 7.0, F32_EXTRA = 20.0, MANY_EXTRA = 33.0;
bool two_passes(const Kv4Att &a, int groups, int nsm) {
    long long keys = a.shared_S;
    if (a.window && keys > (long long)a.window + a.sinks) keys = (long long)a.window + a.sinks;
    auto work = [&](int sequences, long long rows) {
        if (many_rows(a.f32, sequences, a.H, (int)(rows / a.G), a.G)) {
            const long long rest = rows % 256;
            return 2.1 / 6 * (rows / 256 * 6 + (rest == 0 ? 0 : rest <= 128 ? 4 : 6)) * sequences * a.H * (keys / 128.0) / nsm;
        }
        return (a.f32 ? 5.2 : 1.75) * ((rows + 15) / 16) * sequences * a.H * (keys / 256.0) / (2.0 * nsm);
    };
    const long long rows = (long long)a.n * a.G;
    const bool many = many_rows(a.f32, a.B, a.H, a.n, a.G);
    return work(a.B, rows) - work(groups, rows * a.per) > (many ? MANY_EXTRA : a.f32 ? F32_EXTRA : FEW_EXTRA);
}

#ifdef ACES_CHECKED
int forced_passes = 0, last_passes = 0;  // of kv4_shared_attention; not for calls from several threads
#endif

}  // namespace

extern "C" {

int aces_kv4_row_bytes(int D) { return D == 64 || D == 128 ? kv4_row_bytes(D) : -1; }

aces_status aces_kv4_append(void *cache, int planes, int layer, int B, int H, int S, int D, const void *k, const void *v,
                            aces_dtype dt, const int64_t *k_strides, const int64_t *v_strides, const int32_t *start,
                            const int32_t *count, int n, int32_t *row_status, aces_stream_t stream) {
    Kv4Rows a;
    aces_status st = check_cache(cache, planes, layer, B, H, S, D, &a.k, &a.v);
    if (st != ACES_OK) return st;
    st = check_rows(k, v, dt, start, B, n, H);
    if (st != ACES_OK) return st;
    if (!row_status || !k_strides || !v_strides) return ACES_ERR_INVALID_ARG;
    a.f32 = dt == ACES_F32;
    const size_t es = a.f32 ? 4 : 2;
    a.vec = on_grid(k, k_strides, es) && on_grid(v, v_strides, es);
    a.xk = const_cast<void *>(k);
    a.xv = const_cast<void *>(v);
    a.kb = k_strides[0], a.ki = k_strides[1], a.kh = k_strides[2];
    a.vb = v_strides[0], a.vi = v_strides[1], a.vh = v_strides[2];
    a.start = start;
    a.count = count;
    a.status = row_status;
    a.B = B, a.n = n, a.H = H, a.S = S, a.D = D;
    return launch_kv4_append(a, sm_count(), reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? ACES_OK : ACES_ERR_CUDA;
}

aces_status aces_kv4_read(const void *cache, int planes, int layer, int B, int H, int S, int D, const int32_t *start, int n,
                          void *k, void *v, aces_dtype dt, aces_stream_t stream) {
    Kv4Rows a;
    aces_status st = check_cache(cache, planes, layer, B, H, S, D, &a.k, &a.v);
    if (st != ACES_OK) return st;
    st = check_rows(k, v, dt, start, B, n, H);
    if (st != ACES_OK) return st;
    if (!aligned16(k) || !aligned16(v)) return ACES_ERR_INVALID_ARG;
    a.f32 = dt == ACES_F32;
    a.vec = 1;
    a.xk = k;
    a.xv = v;
    a.kb = a.ki = a.kh = a.vb = a.vi = a.vh = 0;
    a.start = start;
    a.count = nullptr;
    a.status = nullptr;
    a.B = B, a.n = n, a.H = H, a.S = S, a.D = D;
    return launch_kv4_read(a, sm_count(), reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? ACES_OK : ACES_ERR_CUDA;
}

size_t aces_kv4_workspace_bytes(int B, int n, int Hq, int H, int D) {
    if (B < 1 || n < 1 || H < 1 || Hq < H || Hq % H != 0 || (D != 64 && D != 128)) return 0;
    if ((long long)B * n > INT_MAX / 2 || (long long)B * n * Hq > INT_MAX / 2) return 0;
    const int G = Hq / H, nsm = sm_count();  // of either type
    const size_t few = kv4_few_ws(n, G, D, nsm), many = many_rows(0, B, H, n, G) ? kv4_many_ws(n, G, D, nsm) : 0;
    return few > many ? few : many;
}

aces_status aces_kv4_attention(const void *q, aces_dtype dt, const int64_t *q_strides, const void *cache, int planes,
                               int layer, int B, int n, int Hq, int H, int S, int D, const int32_t *prefix_len,
                               const int32_t *count, const uint32_t *mask, int64_t mask_stride, const int32_t *depth,
                               int64_t depth_stride, float scale, int window, int sinks, void *out, float *lse,
                               int32_t *seq_status, void *workspace, size_t workspace_bytes, aces_stream_t stream) {
    uint8_t *pk, *pv;
    aces_status st = check_cache(cache, planes, layer, B, H, S, D, &pk, &pv);
    if (st != ACES_OK) return st;
    Kv4Att a;
    st = check_attention(q, dt, q_strides, B, n, Hq, H, D, prefix_len, mask, mask_stride, depth, depth_stride, scale, window, sinks, out,
                         seq_status, workspace, &a);
    if (st != ACES_OK) return st;
    const size_t need = aces_kv4_workspace_bytes(B, n, Hq, H, D);
    if (need == 0 || workspace_bytes < need) return ACES_ERR_INVALID_ARG;
    a.k = pk, a.v = pv, a.S = S;
    a.lse = lse, a.count = count;
    const auto launch = many_rows(a.f32, B, H, n, a.G) ? launch_kv4_many<KV4_ALONE> : launch_kv4_few<KV4_ALONE>;
    return launch(a, workspace, sm_count(), reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? ACES_OK : ACES_ERR_CUDA;
}

// Workspace of two passes: the first's sums, maxima, sums of weights and status, then what
// each pass needs for itself.
static size_t shared_part_bytes(int B, int groups, int n, int Hq, int D) {
    return (size_t)B * n * Hq * (D + 2) * 4 + ((size_t)groups * 4 + 15) / 16 * 16;
}
size_t aces_kv4_shared_workspace_bytes(int B, int groups, int n, int Hq, int H, int D) {
    if (groups < 1 || B < groups || B % groups != 0) return 0;
    const size_t own = aces_kv4_workspace_bytes(B, n, Hq, H, D);
    if (own == 0) return 0;
    const size_t first = aces_kv4_workspace_bytes(groups, B / groups * n, Hq, H, D);
    return (shared_part_bytes(B, groups, n, Hq, D) + 15) / 16 * 16 + (first + 15) / 16 * 16 + own;
}

aces_status aces_kv4_shared_attention(const void *q, aces_dtype dt, const int64_t *q_strides, const void *shared, int shared_planes,
                                      int groups, int S0, const int32_t *shared_len, const void *cache, int planes, int layer, int B,
                                      int n, int Hq, int H, int S, int D, const int32_t *prefix_len, const int32_t *count,
                                      const uint32_t *mask, int64_t mask_stride, const int32_t *depth, int64_t depth_stride, float scale,
                                      int window, int sinks, void *out, float *lse, int32_t *seq_status, void *workspace,
                                      size_t workspace_bytes, aces_stream_t stream) {
    uint8_t *pk, *pv, *sk, *sv;
    aces_status st = check_cache(cache, planes, layer, B, H, S, D, &pk, &pv);
    if (st != ACES_OK) return st;
    if (groups < 1 || B < groups || B % groups != 0) return ACES_ERR_INVALID_ARG;
    st = check_cache(shared, shared_planes, layer, groups, H, S0, D, &sk, &sv);
    if (st != ACES_OK) return st;
    if (!shared_len) return ACES_ERR_INVALID_ARG;
    Kv4Att a;
    st = check_attention(q, dt, q_strides, B, n, Hq, H, D, prefix_len, mask, mask_stride, depth, depth_stride, scale, window, sinks, out,
                         seq_status, workspace, &a);
    if (st != ACES_OK) return st;
    const size_t need = aces_kv4_shared_workspace_bytes(B, groups, n, Hq, H, D);
    if (need == 0 || workspace_bytes < need) return ACES_ERR_INVALID_ARG;
    const int per = B / groups;
    const size_t rows = (size_t)B * n * Hq;
    a.lse = lse, a.count = count, a.per = per;
    a.part = reinterpret_cast<float *>(workspace);
    a.part_m = a.part + rows * D;
    a.part_l = a.part_m + rows;
    a.part_status = reinterpret_cast<int32_t *>(a.part_l + rows);
    a.shared_len = shared_len, a.shared_S = S0;
    uint8_t *first_ws = reinterpret_cast<uint8_t *>(workspace) + (shared_part_bytes(B, groups, n, Hq, D) + 15) / 16 * 16;
    uint8_t *own_ws = first_ws + (aces_kv4_workspace_bytes(groups, per * n, Hq, H, D) + 15) / 16 * 16;  // the passes run side by side
    Kv4Att f = a;
    f.k = sk, f.v = sv;
    f.B = groups, f.n = per * n, f.S = S0;
    f.prefix = shared_len, f.count = nullptr, f.status = a.part_status;
    f.own_n = n, f.own_S = S, f.own_prefix = prefix_len, f.own_count = count;
    a.k = pk, a.v = pv, a.S = S;
    const int nsm = sm_count();
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    bool two = two_passes(a, groups, nsm);
#ifdef ACES_CHECKED
    if (forced_passes) two = forced_passes == 2;
    last_passes = two ? 2 : 1;
#endif
    if (!two) {
        a.k0 = sk, a.v0 = sv;
        const auto split = many_rows(a.f32, B, H, n, a.G) ? launch_kv4_many<KV4_SPLIT> : launch_kv4_few<KV4_SPLIT>;
        return split(a, own_ws, nsm, s) == cudaSuccess ? ACES_OK : ACES_ERR_CUDA;
    }
    const auto first = many_rows(f.f32, f.B, H, f.n, f.G) ? launch_kv4_many<KV4_FIRST> : launch_kv4_few<KV4_FIRST>;
    const auto behind = many_rows(a.f32, B, H, n, a.G) ? launch_kv4_many<KV4_BEHIND> : launch_kv4_few<KV4_BEHIND>;
    if (first(f, first_ws, nsm, s) != cudaSuccess) return ACES_ERR_CUDA;
    return behind(a, own_ws, nsm, s) == cudaSuccess ? ACES_OK : ACES_ERR_CUDA;
}

aces_status aces_rotate_qk(const void *q, const void *k, aces_dtype dt, const int64_t *q_strides, const int64_t *k_strides, int B, int n,
                           int Hq, int H, int D, const aces_turn *turn, void *q_out, void *k_out, const int64_t *q_out_strides,
                           const int64_t *k_out_strides, aces_stream_t stream) {
    Turn a = {};
    const aces_status st = check_turn(turn, D, B, n, Hq, H, q, k, dt, &a);
    if (st != ACES_OK) return st;
    const size_t es = dt == ACES_F32 ? 4 : 2;
    if (!q_out || !k_out || !q_strides || !k_strides || !q_out_strides || !k_out_strides) return ACES_ERR_INVALID_ARG;
    if ((uintptr_t)q_out % es || (uintptr_t)k_out % es) return ACES_ERR_INVALID_ARG;
    if (!apart(q_out_strides, B, n, Hq, D) || !apart(k_out_strides, B, n, H, D)) return ACES_ERR_INVALID_ARG;
    if (!turn->positions && !turn->start) return ACES_ERR_INVALID_ARG;
    a.q = heads(q, q_strides), a.k = heads(k, k_strides);
    a.oq = heads(q_out, q_out_strides), a.ok = heads(k_out, k_out_strides);
    a.vec = on_grid(q, q_strides, es) && on_grid(k, k_strides, es) && on_grid(q_out, q_out_strides, es) && on_grid(k_out, k_out_strides, es);
    return launch_turn(a, D, dt == ACES_F32, false, turn->interleaved != 0, sm_count(), reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess
               ? ACES_OK
               : ACES_ERR_CUDA;
}

aces_status aces_kv4_append_rotated(void *cache, int planes, int layer, int B, int H, int S, int D, const void *q, const void *k,
                                    const void *v, aces_dtype dt, const int64_t *q_strides, const int64_t *k_strides,
                                    const int64_t *v_strides, int Hq, const int32_t *start, const int32_t *count, int n,
                                    const aces_turn *turn, void *q_out, const int64_t *q_out_strides, int32_t *row_status,
                                    aces_stream_t stream) {
    Turn a = {};
    aces_status st = check_cache(cache, planes, layer, B, H, S, D, &a.ck, &a.cv);
    if (st != ACES_OK) return st;
    st = check_turn(turn, D, B, n, Hq, H, q, k, dt, &a);
    if (st != ACES_OK) return st;
    st = check_rows(k, v, dt, start, B, n, H);
    if (st != ACES_OK) return st;
    const size_t es = dt == ACES_F32 ? 4 : 2;
    if (!q_out || !row_status || !q_strides || !k_strides || !v_strides || !q_out_strides || turn->start) return ACES_ERR_INVALID_ARG;
    if ((uintptr_t)q_out % es || !apart(q_out_strides, B, n, Hq, D)) return ACES_ERR_INVALID_ARG;
    a.start = start, a.count = count, a.status = row_status, a.S = S;
    a.q = heads(q, q_strides), a.k = heads(k, k_strides), a.v = heads(v, v_strides), a.oq = heads(q_out, q_out_strides);
    a.vec = on_grid(q, q_strides, es) && on_grid(k, k_strides, es) && on_grid(v, v_strides, es) && on_grid(q_out, q_out_strides, es);
    return launch_turn(a, D, dt == ACES_F32, true, turn->interleaved != 0, sm_count(), reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess
               ? ACES_OK
               : ACES_ERR_CUDA;
}

#ifdef ACES_CHECKED
// How many passes the last aces_kv4_shared_attention took; the next ones take `force` (0: by
// their rule).  For the package's tests: not part of the header.
int aces_checked_shared_passes(int force);
int aces_checked_shared_passes(int force) {
    forced_passes = force;
    return last_passes;
}
#endif

}  // extern "C"
