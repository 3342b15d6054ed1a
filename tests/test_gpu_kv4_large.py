"""The attention over a 4-bit cache at sizes where every SM's ring, places and
pieces are used many times over, against float64 on the GPU, call after call:
what a wait or a fence too few spoils shows here and not in small cases.

Bounds as in test_gpu_kv4.py: 2^-7 (two roundings to bfloat16) and the float32
sums' 4 * 2^-20 (M + 1) + 2^-17 of A, the weights' sum of |v|.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_02514_gb300 as A
    A.load()
    return A


def _seen(P, n, S, mask, depth, window, sinks):
    key = torch.arange(S, device="cuda")[None, :]
    i = torch.arange(n, device="cuda")[:, None]
    t = (key - P).clamp(0, n - 1)
    if mask is None:
        ok, at, pos = key <= P + i, key, P + i
    else:
        ok = (key < P) | (mask[i.expand(n, S), t.expand(n, S)] & (key < P + n))
        at, pos = torch.where(key >= P, P + depth[t], key), P + depth[:, None]
    if window:
        ok = ok & ((at > pos - window) | (at < sinks))
    return ok


def _check(out, lse, q, K, V, ok, scale):
    x = torch.where(ok, (q @ K.T) * scale, -math.inf)
    z = torch.logsumexp(x, -1)
    w = torch.exp(x - z[:, None])
    M = torch.where(ok, (q.abs() @ K.abs().T) * scale, 0.0).amax(1)
    rel = 2.0 ** -7 + 2.0 ** -17 + 4 * 2.0 ** -20 * (M + 1)
    assert ((out.double() - w @ V).abs() <= rel[:, None] * (w @ V.abs())).all()
    assert ((lse.double() - z).abs() <= 2.0 ** -19 * (M + z.abs() + 1)).all()


# B, n (0: the tree of 16 main tokens and 64 branches), Hq, H, D, longest prefix, window, sinks
@pytest.mark.parametrize("B,n,Hq,H,D,P,window,sinks", [
    (8, 0, 32, 8, 128, 5000, 0, 0), (8, 0, 32, 8, 64, 5000, 0, 0), (12, 0, 8, 4, 128, 3000, 0, 0),
    (2, 1500, 16, 4, 128, 2500, 0, 0), (2, 1500, 8, 8, 64, 2500, 0, 0), (3, 1100, 8, 4, 128, 4000, 700, 4), (3, 1100, 8, 4, 64, 4000, 700, 4),
    (40, 1, 32, 8, 128, 8000, 0, 0), (40, 1, 8, 8, 64, 8000, 0, 0), (24, 3, 16, 4, 128, 6000, 0, 0),
])
def test_large_calls_stay_right(A, B, n, Hq, H, D, P, window, sinks):
    gen = torch.Generator(device="cuda").manual_seed(B + n + D)
    mask = depth = words = None
    if n == 0:
        words, depth = A.tree_mask([4] * 16, 1)
        n = depth.numel()
        bits = (words[:, :, None].long() >> torch.arange(32, device="cuda")) & 1
        mask = bits.flatten(1)[:, :n].bool()
    S = P + n
    cache = A.kv4_cache(1, B, H, S, D)
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    for b0 in range(0, S, 2000):
        m = min(2000, S - b0)
        k, v = (torch.randn(B, m, H, D, generator=gen, device="cuda").bfloat16() for _ in range(2))
        A.kv4_append(cache, 0, k, v, zero + b0)
    prefix = torch.tensor([P - (b * 373) % (P // 2) for b in range(B)], dtype=torch.int32, device="cuda")
    q = torch.randn(B, n, Hq, D, generator=gen, device="cuda").bfloat16()
    kv = A.kv4_read(cache, 0, zero, S, dtype=torch.float32)
    first = None
    for rep in range(4):
        r = A.kv4_attention(q, cache, 0, prefix, mask=words, depth=depth, window=window, sinks=sinks)
        torch.cuda.synchronize()
        assert not r["status"].any()
        if first is None:
            first = r
            for b in range(B):
                ok = _seen(int(prefix[b]), n, S, mask, depth, window, sinks)
                for h in range(H):
                    K, V = kv["k"][b, :, h].double(), kv["v"][b, :, h].double()
                    for g in range(h * Hq // H, (h + 1) * Hq // H):
                        _check(r["out"][b, :, g], r["lse"][b, :, g], q[b, :, g].double(), K, V, ok, D ** -0.5)
        assert torch.equal(r["out"], first["out"]) and torch.equal(r["lse"], first["lse"])
