"""Norms of rows whose squares pass float32 and of which one number outweighs the others: the
others' squares are just below half a unit of the sum, and a sum that met them one
after another would lose them all.

Units u = 2^-24.  With position 0, no weights and no scale a rotated number is x / norm alone.
Squares go into eight sums of a lane's 16 numbers (2 u: a product, a fused add), which are
added in three levels, and those of eight (D = 128) or four lanes (D = 64) in three or two more:
8 u at most, half of which shows in the root; the mean with eps 0.5 u, the root 1.5 u, its
product with the number 1 u: 7 u of the number.  The cache's codes are those of the
64-bit numbers, bit for bit.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import turn as O  # noqa: E402
from tests.test_gpu_turn import A, DT, _f64, _freq, _i32  # noqa: E402, F401


def _rows(rng, shape, D, first):
    """Numbers of just below 2^52, one of 2^64 at one of the channels `first` of each row."""
    x = 2.0 ** 52 * (1 - rng.integers(1, 4, shape + (D,)) / 128.0) * rng.choice([-1.0, 1.0], shape + (D,))
    np.put_along_axis(x, rng.choice(first, shape + (1,)), 2.0 ** 64, -1)
    return x


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_rotation_keeps_small_squares(A, D, inter):  # noqa: F811
    rng = np.random.default_rng(D)
    x = torch.from_numpy(_rows(rng, (2, 200, 4), D, np.arange(0, D, 4)).astype(np.float32)).cuda()
    r = A.rotate_qk(x[:, :, :3], x[:, :, 3:], _freq(D), positions=_i32(np.zeros((2, 200))), eps=1e-6, interleaved=inter)
    for got, given in ((r["q"], x[:, :, :3]), (r["k"], x[:, :, 3:])):
        z, _ = O.turned(_f64(given), _f64(_freq(D)), np.zeros((1, 2, 200)), eps=1e-6)
        assert (np.abs(_f64(got) - z) <= 7 * 2.0 ** -24 * np.abs(z)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_codes_of_rows_with_an_outlier(A, D, inter, dtype):  # noqa: F811
    """Each head's weights put its numbers 18 to 22 units below the border of the outermost codes, where a
    norm that lost 31 squares of a lane, 15.4 units, and the other roundings may take them across it."""
    rng = np.random.default_rng(D + inter)
    H, G, pos, eps, scale = 16384, D // 8, 1, 1e-6, 1 + 1.01 * 2.0 ** -24
    x = 2.0 ** 52 * (1 - rng.integers(1, 65, (H, D)) / 256.0)
    lane = np.arange(D) // G < 2 if inter else np.arange(D) // G % 4 == 0
    x[:, lane] = 2.0 ** 52 * 255 / 256
    x *= rng.choice([-1.0, 1.0], x.shape)
    x[:, 0] = 2.0 ** 64
    f = torch.linspace(0.02, 0.1, D // 2, device="cuda")
    k = torch.from_numpy(x.astype(np.float32)).to(DT[dtype]).cuda()[None, None]
    partner = np.arange(D) % 2 == 1 if inter else np.arange(D) >= D // 2
    one = np.where(partner, 0.0, 1.0)                          # z_u = y_u cos, z_v = y_u sin
    at = np.array([[[pos]]])
    z = O.turned(_f64(k), _f64(f), at, None, one, eps, inter, scale)[0][0, 0]
    top = 1.0325 * 2.0 ** -8                                   # of a group: its step is a 7.76th
    step = np.rint(top * 2.0 ** 12) * 2.0 ** -12 / 8
    goal = 7.5 * step * (1 - rng.uniform(18, 22, (H, D)) * 2.0 ** -24)
    goal.reshape(H, 8, G)[:, :, 2] = top
    with np.errstate(divide="ignore"):
        w = torch.from_numpy(np.where(partner, 0.0, goal / z).astype(np.float32)).cuda()
    cache = A.kv4_cache(1, 1, H, 1, D)
    r = A.kv4_append_rotated(cache, 0, k[:, :, :1], k, k, _i32([0]), f, positions=_i32([[pos]]), k_weight=w, eps=eps, interleaved=inter, scale=scale)
    z, _ = O.turned(_f64(k), _f64(f), at, None, _f64(w), eps, inter, scale)
    np.testing.assert_array_equal(_f64(A.kv4_read(cache, 0, _i32([0]), 1, dtype=torch.float32)["k"]), O.held(z))
    assert not r["status"].any()
