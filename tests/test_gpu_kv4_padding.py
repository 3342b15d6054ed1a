"""Attention of many rows where most items have no keys: batches in which a few
sequences have tokens among hundreds that are padding, and prompts of which most
row tiles are.  A CTA then goes through several items without keys in a row, right
after one whose two groups of rows take very different times (the second group's
tokens lie behind the window in the tree's own depths).  Bounds as in test_gpu_kv4.py.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import A, _compare, _f64, _i32, _torch, _words  # noqa: E402, F401


def _run(A, B, n, Hq, H, D, P, cnt, **seen):  # noqa: F811
    """A call on B sequences and its comparison; P and cnt by sequence."""
    rng = np.random.default_rng(B + n + D)
    S = max(P) + n
    live = [b for b in range(B) if cnt[b] > 0]
    cache = A.kv4_cache(1, B, H, S, D)
    kv = {}
    for b in live:
        kv[b] = [rng.standard_normal((1, S, H, D)) for _ in range(2)]
        one = A.kv4_cache(1, 1, H, S, D)
        A.kv4_append(one, 0, *(_torch(x, "f32") for x in kv[b]), _i32([0]))
        cache[:, b] = one[:, 0]
        back = A.kv4_read(one, 0, _i32([0]), S, dtype=torch.float32)
        kv[b] = [_f64(back[k]).swapaxes(1, 2) for k in ("k", "v")]
    gen = torch.Generator(device="cuda").manual_seed(n)
    q = torch.randn(B, n, Hq, D, generator=gen, device="cuda").bfloat16()
    mask, depth = seen.pop("mask", None), seen.pop("depth", None)
    r = A.kv4_attention(q, cache, 0, _i32(P), count=_i32(cnt), mask=None if mask is None else _words(mask),
                        depth=None if depth is None else _i32(depth), **seen)
    torch.cuda.synchronize()
    assert not r["status"].any()
    none = torch.tensor([c == 0 for c in cnt], device="cuda")
    assert not r["out"][none].any() and torch.isneginf(r["lse"][none]).all()
    for b in live:
        _compare({k: r[k][b:b + 1] for k in ("out", "lse")}, _f64(q[b:b + 1]), *kv[b], [P[b]], [cnt[b]], "bf16", D ** -0.5, mask, depth, **seen)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,n,every", [(1500, 32, 97), (1500, 16, 97), (700, 40, 31), (300, 32, 300)])
def test_padding_after_uneven_groups(A, D, B, n, every):  # noqa: F811
    Hq, H = 8, 1
    mask = np.tril(np.ones((n, n), bool))
    depth = np.where(np.arange(n) < n // 2, 0, 100 + np.arange(n))   # the second half lies behind the window
    P = [300 + (b * 53) % 400 if b % every == 0 else 0 for b in range(B)]
    cnt = [n if b % every == 0 else 0 for b in range(B)]
    _run(A, B, n, Hq, H, D, P, cnt, mask=mask, depth=depth, window=60, sinks=2)


@pytest.mark.parametrize("D", [64, 128])
def test_prompts_that_are_mostly_padding(A, D):  # noqa: F811
    _run(A, 6, 1500, 4, 2, D, [100, 0, 700, 3, 0, 260], [40, 0, 300, 1, 0, 7])


def test_nothing_but_padding(A):  # noqa: F811
    _run(A, 400, 50, 4, 2, 64, [0] * 399 + [9], [0] * 400)
