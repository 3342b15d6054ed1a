"""Shared prefixes, rotated rows and queries past 2^32 bytes: of a prefix's plane, of the
cache that is written, of the strided arrays that are read and written.  Bounds as in
test_gpu_kv4.py and test_gpu_turn.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import turn as O  # noqa: E402
from tests.test_gpu_kv4 import A, _compare, _f64, _filled, _i32, _torch  # noqa: E402, F401

G, H, Hq, D, S0, BACK = 65, 1, 2, 128, 830000, 4100


def _room(gb):
    if torch.cuda.mem_get_info()[0] < gb << 30:
        pytest.skip(f"needs {gb} GB of device memory")


@pytest.fixture(scope="module")
def far(A):  # noqa: F811
    _room(40)
    shared = torch.empty(4, G, H, S0, D // 2 + 16, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(9)
    at = S0 - 7                                              # the last prefix's length
    assert ((G - 1) * S0 + at - BACK) * (D // 2 + 16) > 1 << 32
    start = _i32([0] * (G - 1) + [at - BACK])
    k, v = (torch.randn(G, BACK, H, D, generator=gen, device="cuda") for _ in range(2))
    A.kv4_append(shared, 1, k, v, start)
    back = A.kv4_read(shared, 1, start, BACK, dtype=torch.float32)
    K, V = (_f64(back[x][G - 1:]).swapaxes(1, 2) for x in ("k", "v"))
    yield shared, K, V, _i32([0] * (G - 1) + [at])
    del shared
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("per,n,window", [(1, 1, 4000), (2, 1, 64), (20, 1, 4000), (1, 40, 500), (2, 40, 4000)])
def test_far_prefixes(A, far, per, n, window, dtype):  # noqa: F811
    shared, K0, V0, lens = far
    rng = np.random.default_rng(per + n)
    B = G * per
    cache, K, V = _filled(A, rng, B, H, 3 + n, D, layers=2, layer=1)
    q = _torch(rng.standard_normal((B, n, Hq, D)), dtype)
    r = A.kv4_shared_attention(q, shared, lens, cache, 1, _i32([3] * B), window=window)
    assert not r["status"].any()
    for b in (B - per, B - 1):      # of the last prefix; positions counted from BACK before its end
        Kb, Vb = (np.concatenate([s, o[b:b + 1]], 2) for s, o in ((K0, K), (V0, V)))
        _compare({x: r[x][b:b + 1] for x in ("out", "lse")}, _f64(q[b:b + 1]), Kb, Vb, [BACK + 3], [n], dtype, D ** -0.5, window=window)


def test_far_rows_are_turned_and_written(A):  # noqa: F811
    _room(60)
    B, n, Hk = 2, 5, 2
    S = (1 << 32) // ((D // 2 + 16) * Hk) + 100               # the second sequence's rows begin past 2^32 bytes
    rng = np.random.default_rng(3)
    wide = torch.empty((1 << 32) + 4096 * 64, dtype=torch.bfloat16, device="cuda")
    step = (1 << 32) // 8 * 8                                  # numbers between the two sequences'
    qkv = wide.as_strided((B, n, 4 + 2 * Hk, D), (step, 8 * (4 + 2 * Hk) * D, D, 1))
    qkv.copy_(torch.from_numpy(rng.standard_normal(qkv.shape).astype(np.float32)))
    q, k, v = qkv.split([4, Hk, Hk], dim=2)
    q64, k64, v64 = _f64(q), _f64(k), _f64(v)
    f = torch.from_numpy((10000.0 ** (-np.arange(64) / 64)).astype(np.float32)).cuda()
    cache = torch.empty(2, B, Hk, S, D // 2 + 16, dtype=torch.uint8, device="cuda")
    start = np.array([S - n, S - n - 1])
    r = A.kv4_append_rotated(cache, 0, q, k, v, _i32(start), f, eps=1e-6, out=dict(q=q))
    assert r["q"] is q and not r["status"].any()
    pos = (start[:, None] + np.arange(n))[None]
    z, h = O.turned(q64, _f64(f), pos, eps=1e-6)
    assert (np.abs(_f64(q) - z) <= 16 * 2.0 ** -24 * h * 1.01 + 2.0 ** -8 * np.abs(z)).all()
    back = A.kv4_read(cache, 0, _i32(start), n, dtype=torch.float32)
    np.testing.assert_array_equal(_f64(back["k"]), O.held(O.turned(k64, _f64(f), pos, eps=1e-6)[0]))
    np.testing.assert_array_equal(_f64(back["v"]), O.held(v64))
    r = A.rotate_qk(q, k, f, start=_i32([0, 0]))              # far inputs to near outputs
    z, h = O.turned(k64, _f64(f), np.broadcast_to(np.arange(n), (1, B, n)))
    assert (np.abs(_f64(r["k"]) - z) <= 16 * 2.0 ** -24 * h * 1.01 + 2.0 ** -8 * np.abs(z)).all()
    del wide, cache
    torch.cuda.empty_cache()
