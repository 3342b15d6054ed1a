"""Float32 queries keep all their 24 bits, and so do the weights: bounds that two
bfloat16 parts instead of three would not meet (the second half of each test: the
mistake planted in the reference).

Queries have one channel that is not zero, so a score is one product, in three exact
parts.  Its sum adds them in three steps, each of which cuts off up to two units of
2^-23; the scale, the logarithms' constant and the maximum round once each, 2^-24.
With the exponential and the logarithm of a sum near 1, 2^-22 each at most:
    |lse - s| <= 2^-20 |s| + 2^-21
where one key is seen.  Where two are, with scores 0 and -x, x <= 1/4, and values 0
and v, the result is v w, w = e^-x / (1 + e^-x); relative to it: x 2^-20 <= 2^-22 from
the score, 2^-22 from the exponential, three steps of two units in the product, 2^-23
each from the weights' sum, the division and the result: in all below 2^-19.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import A, _f64, _i32, _torch  # noqa: E402, F401


def _two_parts(x):
    """Numbers as the sum of their first two bfloat16 parts, rounded to nearest."""
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32))
    hi = t.bfloat16().float()
    return (hi + (t - hi).bfloat16().float()).double().numpy()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [8, 3000])                     # a CTA a key head; shares and a join
@pytest.mark.parametrize("G", [1, 12])
def test_queries_keep_their_bits(A, D, S, G):  # noqa: F811
    B, H = 200, 1
    rng = np.random.default_rng(D + G)
    k, v = rng.standard_normal((B, 1, H, D)), rng.standard_normal((B, 1, H, D))
    cache = A.kv4_cache(1, B, H, S, D)
    zero = _i32([0] * B)
    A.kv4_append(cache, 0, _torch(k, "f32"), _torch(v, "f32"), zero)
    K = _f64(A.kv4_read(cache, 0, zero, 1, dtype=torch.float32)["k"])[:, 0, 0]
    at = rng.integers(0, D, (B, G))
    x = (rng.uniform(8, 16, (B, G)) * rng.choice([-1, 1], (B, G))).astype(np.float32).astype(np.float64)
    q = np.zeros((B, 1, G, D))
    np.put_along_axis(q[:, 0], at[..., None], x[..., None], -1)
    r = A.kv4_attention(_torch(q, "f32"), cache, 0, zero, scale=0.5)
    kk = np.take_along_axis(K, at, -1)
    s = 0.5 * x * kk
    bound = 2.0 ** -20 * np.abs(s) + 2.0 ** -21
    assert (np.abs(_f64(r["lse"])[:, 0] - s) <= bound).all()
    assert not (np.abs(0.5 * _two_parts(x) * kk - s) <= bound).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [8, 3000])
@pytest.mark.parametrize("G", [1, 12])
def test_weights_keep_their_bits(A, D, S, G):  # noqa: F811
    B, H = 200, 1
    rng = np.random.default_rng(D + G)
    k, v = rng.standard_normal((B, 2, H, D)), rng.standard_normal((B, 2, H, D))
    k[:, 0] = v[:, 0] = 0.0                                  # position 0: score 0, value 0
    k[:, 1, :, 0] = -8.0                                     # held as it is, with a step of 1
    cache = A.kv4_cache(1, B, H, S, D)
    zero = _i32([0] * B)
    A.kv4_append(cache, 0, _torch(k, "f32"), _torch(v, "f32"), zero)
    back = A.kv4_read(cache, 0, zero, 2, dtype=torch.float32)
    K, V = (_f64(back[x])[:, :, 0] for x in ("k", "v"))
    assert (K[:, 1, 0] == -8.0).all() and not K[:, 0].any() and not V[:, 0].any()
    x = rng.uniform(0.01, 0.25, (B, G)).astype(np.float32)
    q = np.zeros((B, 1, G, D))
    q[:, 0, :, 0] = x / 8
    r = A.kv4_attention(_torch(q, "f32"), cache, 0, zero + 1, scale=1.0)
    p = np.exp(-x.astype(np.float64))
    want = (p / (1 + p))[..., None] * V[:, 1][:, None]
    out = _f64(r["out"])[:, 0]
    assert (np.abs(out - want) <= 2.0 ** -19 * np.abs(want)).all()
    assert (np.abs(_f64(r["lse"])[:, 0] - np.log1p(p)) <= 2.0 ** -19).all()
    short = (_two_parts(p) / (1 + p))[..., None] * V[:, 1][:, None]
    assert not (np.abs(short - want) <= 2.0 ** -19 * np.abs(want)).all()
