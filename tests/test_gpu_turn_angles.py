"""Angles up to 2^40: t = p * inv_freq is a product in 64 bits, whose rounding shows from some 2^29
on, and whole turns fall off whatever their number.  Bounds are test_gpu_turn.py's, and the cache's codes
are those of the 64-bit numbers."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import turn as O  # noqa: E402
from tests.test_gpu_turn import A, DT, _close, _f64, _i32  # noqa: E402, F401


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_angles_up_to_2_to_the_40(A, D, inter, dtype):  # noqa: F811
    rng = np.random.default_rng(D + inter)
    n, H = 400, 2
    x = torch.from_numpy(rng.standard_normal((1, n, 3 * H, D)).astype(np.float32)).to(DT[dtype]).cuda()
    q, k, v = x.split([H, H, H], dim=2)
    # of two halves of the pairs: slow ones at any position, fast ones up to 2^40 / f of their own axis
    f = rng.choice([-1.0, 1.0], D // 2) * 2.0 ** rng.uniform(-100, 9, D // 2)
    fast = rng.random(D // 2) < 0.5
    f[fast] = rng.choice([-1.0, 1.0], fast.sum()) * 2.0 ** rng.uniform(9, 29, fast.sum())
    f[:8], fast[:8] = [1.0, -1.0, 0.9, 400.0, 1e6, 2.0 ** 28, 0.0, 1e-45], [False] * 4 + [True, True] + [False] * 2
    f = torch.from_numpy(f.astype(np.float32)).cuda()
    pos = np.sign(rng.standard_normal((2, n))) * np.floor(2.0 ** (rng.uniform(0, 1, (2, n)) * [[31], [11]]))
    pos[0, :5] = [2 ** 31 - 1, -2 ** 31, 0, 2 ** 26, 1]
    at, axes = pos[:, None], fast.astype(np.int32)
    where = dict(positions=_i32(at), axes=_i32(axes), interleaved=inter)
    r = A.rotate_qk(q, k, f, **where)
    for got, given in ((r["q"], q), (r["k"], k)):
        z, h = O.turned(_f64(given), _f64(f), at, axes, interleaved=inter)
        _close(got, z, h, dtype)
    for turn in (dict(), dict(eps=1e-6)):
        cache = A.kv4_cache(1, 1, H, n, D)
        r = A.kv4_append_rotated(cache, 0, q, k, v, _i32([0]), f, **where, **turn)
        z, h = O.turned(_f64(q), _f64(f), at, axes, interleaved=inter, **turn)
        _close(r["q"], z, h, dtype)
        z, _ = O.turned(_f64(k), _f64(f), at, axes, interleaved=inter, **turn)
        np.testing.assert_array_equal(_f64(A.kv4_read(cache, 0, _i32([0]), n, dtype=torch.float32)["k"]), O.held(z))
        assert not r["status"].any()
