"""Attention of many rows behind 600 thousand positions that one CTA has alone, with
values of one sign: what the tensor cores' sums cut off would all lie on one side.

Bound of the mean relative distance to float64, over 24 key heads, 64 channels and all
rows: 1024 adds between two totals, each at most a unit (2^-23) low, are 2^-13; the
results' rounding to bfloat16 has a standard deviation of at most 2^-7 / sqrt(12) =
0.0023 a number, 0.000058 for the mean over 24 * 64 channels (a head's rows round
alike), and four of those are below 2^-12.  Without totals the sums would lie some
600000 / 16 / 2 units, 0.0011 of 2^0, low.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import A  # noqa: E402, F401


@pytest.mark.parametrize("n,G", [(64, 4), (32, 4)])          # two groups of 128 rows; both on the same 128
def test_long_sums_are_not_cut_off(A, n, G):  # noqa: F811
    B, H, D, S = 19, 8, 64, 600000
    free, _ = torch.cuda.mem_get_info()
    if free < 30 << 30:
        pytest.skip("needs 30 GB of device memory")
    gen = torch.Generator(device="cuda").manual_seed(n)
    cache = A.kv4_cache(1, B, H, S, D)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    looked = [(b, h) for b in (0, 9, 18) for h in range(H)]
    for b, h in looked:                                      # the others stay zeros: the same work
        one = A.kv4_cache(1, 1, 1, S, D)
        k = torch.randn(1, S, 1, D, generator=gen, device="cuda")
        v = (torch.rand(1, S, 1, D, generator=gen, device="cuda") + 0.5) * (1 + torch.rand(D, generator=gen, device="cuda"))
        A.kv4_append(one, 0, k, v, zero)
        cache[:, b, h] = one[:, 0, 0]
    q = (0.5 * torch.randn(B, n, H * G, D, generator=gen, device="cuda")).bfloat16()
    r = A.kv4_attention(q, cache, 0, torch.full((B,), S - n, dtype=torch.int32, device="cuda"))
    assert not r["status"].any()
    seen = torch.arange(S, device="cuda")[None] <= S - n + torch.arange(n, device="cuda")[:, None]
    far = []
    for b, h in looked:
        kv = A.kv4_read(cache[:, b:b + 1, h:h + 1].contiguous(), 0, zero, S, dtype=torch.float32)
        K, V = kv["k"][0, :, 0].double(), kv["v"][0, :, 0].double()
        for g in range(h * G, (h + 1) * G):
            x = torch.where(seen, q[b, :, g].double() @ K.T * D ** -0.5, -math.inf)
            z = torch.logsumexp(x, -1)
            want = torch.exp(x - z[:, None]) @ V
            off = (r["out"][b, :, g].double() - want) / want
            assert off.abs().max() <= 2.0 ** -7
            assert ((r["lse"][b, :, g].double() - z).abs() <= 2.0 ** -16).all()
            far.append(off)
    assert abs(float(torch.stack(far).mean())) <= 2.0 ** -13 + 2.0 ** -12
