// C entry points of the 4-bit KV cache: argument checks and launches.
#include <climits>

#include "kv4_plan.cuh"

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
    Kv4Att a;
    uint8_t *pk, *pv;
    aces_status st = check_cache(cache, planes, layer, B, H, S, D, &pk, &pv);
    if (st != ACES_OK) return st;
    if (dt != ACES_F32 && dt != ACES_BF16) return ACES_ERR_UNSUPPORTED;
    if (!q || !q_strides || !prefix_len || !out || !seq_status || !workspace) return ACES_ERR_INVALID_ARG;
    const size_t es = dt == ACES_F32 ? 4 : 2;
    if ((uintptr_t)q % es || !aligned16(out) || !aligned16(workspace)) return ACES_ERR_INVALID_ARG;
    if (n < 1 || Hq < H || Hq % H != 0) return ACES_ERR_INVALID_ARG;
    const size_t need = aces_kv4_workspace_bytes(B, n, Hq, H, D);
    if (need == 0 || workspace_bytes < need) return ACES_ERR_INVALID_ARG;
    if ((mask == nullptr) != (depth == nullptr)) return ACES_ERR_INVALID_ARG;
    const int words = (n + 31) / 32;
    if (mask && ((mask_stride != 0 && mask_stride < (int64_t)n * words) || (depth_stride != 0 && depth_stride < n)))
        return ACES_ERR_INVALID_ARG;
    if (!(scale > 0.0f && scale <= 0x1p110f)) return ACES_ERR_INVALID_ARG;  // a.scale below is finite
    if (window < 0 || sinks < 0) return ACES_ERR_INVALID_ARG;
    a.k = pk, a.v = pv;
    a.q = q;
    a.qb = q_strides[0], a.qi = q_strides[1], a.qh = q_strides[2];
    a.f32 = dt == ACES_F32;
    a.out = out, a.lse = lse, a.status = seq_status;
    a.prefix = prefix_len, a.count = count;
    a.mask = mask, a.mask_b = mask_stride, a.depth = depth, a.depth_b = depth_stride;
    a.B = B, a.n = n, a.Hq = Hq, a.H = H, a.G = Hq / H, a.S = S, a.D = D, a.words = words;
    a.window = window;
    a.sinks = window > 0 ? sinks : 0;
    a.scale = (float)((double)scale * 1.4426950408889634 * (double)KV4_STEP);
    const auto launch = many_rows(a.f32, B, H, n, a.G) ? launch_kv4_many : launch_kv4_few;
    return launch(a, workspace, sm_count(), reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? ACES_OK : ACES_ERR_CUDA;
}

}  // extern "C"
