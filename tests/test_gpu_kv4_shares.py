"""Attention of few rows whose work is shared out and joined, and by one CTA a key
head where there are more of them than SMs: float32, 9 to 16 rows a key head, and
the joins of two or three pieces and of many, against float64 on the GPU.

Bounds as in test_gpu_kv4.py: float32 sums' 4 * 2^-20 (M + 1) + 2^-17 of A, the
weights' sum of |v|, and 2^-7 for bfloat16 queries.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4_large import A, _seen  # noqa: E402, F401

# B, n, Hq, H, longest prefix, window, sinks.  80 key heads take a CTA each up to 2048
# positions of the cache and shares beyond, two key heads clusters of eight up to 16384.
CASES = [
    (40, 1, 8, 2, 2400, 0, 0),
    (40, 3, 8, 2, 2400, 0, 0),          # 12 rows a key head
    (40, 10, 6, 2, 2600, 0, 0),         # 30: two tiles of rows
    (40, 1, 24, 2, 2300, 0, 0),
    (20, 2, 16, 4, 5000, 2500, 3),
    (1, 1, 2, 2, 20000, 0, 0),          # many pieces
    (1, 4, 6, 2, 18000, 0, 0),
    (2, 1, 3, 1, 40000, 0, 0),
    (60, 1, 8, 4, 800, 0, 0),           # 240 key heads, a CTA each
    (60, 4, 12, 4, 800, 0, 0),
    (60, 1, 8, 4, 1900, 0, 0),
    (60, 4, 12, 4, 1900, 0, 0),
]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_shares_and_joins(A, case, dtype, D):  # noqa: F811
    B, n, Hq, H, P, window, sinks = case
    gen = torch.Generator(device="cuda").manual_seed(B + n + D)
    S = P + n
    cache = A.kv4_cache(1, B, H, S, D)
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    k, v = (torch.randn(B, S, H, D, generator=gen, device="cuda") for _ in range(2))
    A.kv4_append(cache, 0, k, v, zero)
    prefix = torch.tensor([P - (b * 373) % (P // 2) for b in range(B)], dtype=torch.int32, device="cuda")
    q = torch.randn(B, n, Hq, D, generator=gen, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    kv = A.kv4_read(cache, 0, zero, S, dtype=torch.float32)
    r = A.kv4_attention(q, cache, 0, prefix, window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert not r["status"].any()
    scale = D ** -0.5
    for b in range(B):
        ok = _seen(int(prefix[b]), n, S, None, None, window, sinks)
        K, V = (kv[x][b].double().transpose(0, 1).repeat_interleave(Hq // H, 0) for x in ("k", "v"))
        qb = q[b].double().transpose(0, 1)
        x = torch.where(ok, (qb @ K.transpose(1, 2)) * scale, -math.inf)
        z = torch.logsumexp(x, -1)
        w = torch.exp(x - z[..., None])
        M = torch.where(ok, (qb.abs() @ K.abs().transpose(1, 2)) * scale, 0.0).amax(-1)
        rel = (2.0 ** -7 if dtype == "bf16" else 0.0) + 2.0 ** -17 + 4 * 2.0 ** -20 * (M + 1)
        out, lse = r["out"][b].double().transpose(0, 1), r["lse"][b].double().transpose(0, 1)
        assert ((out - w @ V).abs() <= rel[..., None] * (w @ V.abs())).all(), b
        assert ((lse - z).abs() <= 2.0 ** -19 * (M + z.abs() + 1)).all(), b
    for _ in range(3):
        again = A.kv4_attention(q, cache, 0, prefix, window=window, sinks=sinks)
        assert torch.equal(r["out"], again["out"]) and torch.equal(r["lse"], again["lse"])
