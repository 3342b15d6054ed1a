"""Attention at the ends of float32's range: queries beyond the largest bfloat16 are
finite numbers like others.  Bounds as in test_gpu_kv4.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import A, _compare, _f64, _i32, _torch  # noqa: E402, F401

FLT_MAX = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,Hq,H,P", [(1, 4, 2, 40), (9, 4, 2, 300), (1, 2, 1, 3000)])
def test_queries_beyond_the_largest_bfloat16(A, n, Hq, H, P, D):  # noqa: F811
    rng = np.random.default_rng(n + D)
    B, S = 1, P + n
    k, v = rng.standard_normal((B, S, H, D)), rng.standard_normal((B, S, H, D))
    k[..., :D // 8] = 0.0                                    # the first group: zeros
    k[..., D // 8:D // 4] *= 1e-25                           # the second: tiny
    cache = A.kv4_cache(1, B, H, S, D)
    A.kv4_append(cache, 0, _torch(k, "f32"), _torch(v, "f32"), _i32([0]))
    back = A.kv4_read(cache, 0, _i32([0]), S, dtype=torch.float32)
    K, V = _f64(back["k"]).swapaxes(1, 2), _f64(back["v"]).swapaxes(1, 2)
    q = rng.standard_normal((B, n, Hq, D))
    q[..., 1] = FLT_MAX
    q[..., 2] = -FLT_MAX * (1 - 2.0 ** -10)
    t = _torch(q, "f32")
    r = A.kv4_attention(t, cache, 0, _i32([P]))
    _compare(r, _f64(t), K, V, [P], [n], "f32", D ** -0.5)
    q[..., D // 8 + 3] = FLT_MAX                             # scores of some 1e13 before the scale
    t = _torch(q, "f32")
    r = A.kv4_attention(t, cache, 0, _i32([P]), scale=1e-14)
    _compare(r, _f64(t), K, V, [P], [n], "f32", 1e-14)
