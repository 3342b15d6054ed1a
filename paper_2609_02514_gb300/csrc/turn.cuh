// Arguments of the rotation of queries and keys (turn.cu).
#pragma once
#include "kv4.cuh"

namespace aces {

struct TurnHeads {  // [B, n, heads, D] numbers, the last dimension dense; strides in elements
    void *p;
    long long b, i, h;
};
struct TurnWeight {
    const void *p;   // null: ones
    long long h;     // between two heads' (0: shared)
    int f32, vec;    // vec: every head's start on 16 bytes
};

struct Turn {
    TurnHeads q, k, v, oq, ok;         // v: append only; ok: rotation only
    int vec;                           // every group starts on 16 bytes
    const float *freq;                 // [R / 2]
    const int32_t *axes;               // [R / 2] or null
    const int32_t *positions;          // [n_axes, B, n] or null
    const int32_t *start, *base, *depth;
    long long depth_b;
    TurnWeight qw, kw;
    int R, n_axes, norm;
    double eps, scale;
    float eps32, eps_low, scale32, scale_low;  // in two parts
    int B, n, Hq, H;
    // append
    uint8_t *ck, *cv;
    const int32_t *count;
    int32_t *status;
    int S;
};
cudaError_t launch_turn(const Turn &a, int D, bool f32, bool append, bool interleaved, int nsm, cudaStream_t s);

}  // namespace aces
