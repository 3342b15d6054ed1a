"""Attention of few rows by a cluster of CTAs a key head, against float64 numpy.

The sizes give clusters of eight, four and two CTAs (by the key heads of all
sequences), some of whose CTAs have no keys, and lengths from nothing to the
last position.  The bounds are test_gpu_kv4's.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import A, _compare, _f64, _filled, _i32, _torch, _tree_bits, _words  # noqa: E402, F401

# B, n, Hq, H, D, positions, lengths, window, sinks
CASES = [
    (1, 1, 8, 2, 128, 4000, [3999], 0, 0),                     # eight CTAs, two steps each
    (1, 1, 8, 2, 128, 4000, [260], 0, 0),                      # keys for two of the eight
    (1, 1, 3, 3, 64, 2100, [0], 0, 0),                         # one key
    (2, 2, 8, 2, 64, 2300, [2298, 511], 0, 0),
    (3, 3, 10, 2, 128, 1500, [1024, 7, 1300], 0, 0),           # 15 rows a key head
    (1, 9, 4, 2, 64, 3000, [2990], 0, 0),                      # 18: two tiles of rows
    (4, 1, 32, 8, 128, 1200, [1199, 600, 33, 0], 0, 0),        # four CTAs
    (8, 1, 16, 8, 64, 900, [899, 800, 700, 512, 256, 255, 31, 1], 0, 0),  # two
    (2, 1, 8, 4, 128, 6000, [5000, 1029], 1024, 4),            # a window in a long cache
    (2, 4, 8, 4, 64, 3300, [3200, 40], 700, 130),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_clusters(A, case, dtype):  # noqa: F811
    B, n, Hq, H, D, S, P, window, sinks = case
    rng = np.random.default_rng(S + n + Hq)
    cache, K, V = _filled(A, rng, B, H, S, D)
    cnt = [n - (b % 2 if n > 1 else 0) for b in range(B)]
    for b in range(B):
        cache[:, b, :, P[b] + cnt[b]:] = 255                    # bytes nobody wrote
    q = _torch(rng.standard_normal((B, n, Hq, D)) * 2.0, dtype)
    r = A.kv4_attention(q, cache, 0, _i32(P), count=_i32(cnt), window=window, sinks=sinks)
    assert not r["status"].any()
    _compare(r, _f64(q), K, V, P, cnt, dtype, D ** -0.5, window=window, sinks=sinks)
    again = A.kv4_attention(q, cache, 0, _i32(P), count=_i32(cnt), window=window, sinks=sinks)
    for key in ("out", "lse"):
        assert torch.equal(r[key], again[key])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_rows_that_see_nothing(A, dtype):  # noqa: F811
    """An empty prefix and mask rows without a bit, next to a sequence outside the cache."""
    rng = np.random.default_rng(11)
    mask, depth = _tree_bits([1, 1], 1)
    n, B, Hq, H, D, S = len(depth), 3, 4, 2, 128, 1800
    masks = np.stack([mask] * B)
    masks[0, 1] = False
    P = [0, 1700, S]
    cache, K, V = _filled(A, rng, B, H, S, D)
    q = _torch(rng.standard_normal((B, n, Hq, D)), dtype)
    r = A.kv4_attention(q, cache, 0, _i32(P), mask=_words(masks), depth=_i32(depth))
    assert r["status"].tolist() == [0, 0, A.ROW_RANGE]
    assert (r["out"][0, 1] == 0).all() and torch.isneginf(r["lse"][0, 1]).all()
    assert (r["out"][2] == 0).all() and torch.isneginf(r["lse"][2]).all()
    _compare({k: r[k][:2] for k in ("out", "lse")}, _f64(q)[:2], K[:2], V[:2], P[:2], [n] * 2, dtype, D ** -0.5, masks[:2], depth)
