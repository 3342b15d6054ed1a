"""Keys into the 4-bit cache at the ends of float32: numbers that are none and those beside
them, products that pass float32 where the 64-bit number does not, weights of any size.
Codes and status are those of the numbers in 64 bits, for every row."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import turn as O  # noqa: E402
from tests.test_gpu_turn import A, DT, _f64, _freq, _i32  # noqa: E402, F401


def _z(x, f, pos, weight=None, eps=None, inter=False, scale=1.0):
    """The definition in real numbers of 64 bits (an infinity times a complex number is more than its parts)."""
    y = np.array(x, np.float64)
    D, half = y.shape[-1], len(f)
    with np.errstate(all="ignore"):
        if eps is not None:
            norm = np.sqrt((y * y).sum(-1, keepdims=True) / D + eps)
            y = (y if weight is None else y * weight) / norm
        z = y.copy()
        for j in range(half):
            u, v = (2 * j, 2 * j + 1) if inter else (j, j + half)
            t = np.asarray(pos, np.float64) * float(f[j])
            c, s = np.cos(t), np.sin(t)
            z[..., u] = scale * (y[..., u] * c - y[..., v] * s)
            z[..., v] = scale * (y[..., v] * c + y[..., u] * s)
    return z


def _step(z):
    g = z.reshape(z.shape[:-1] + (8, -1))
    g = np.where(np.isnan(g), 0.0, np.clip(g, -O.CAP, O.CAP))
    a = np.take_along_axis(g, np.abs(g).argmax(-1)[..., None], -1)
    m, e = np.frexp(a)
    return np.broadcast_to(-np.ldexp(np.rint(m * 32.0), e - 8), g.shape).reshape(z.shape)


def _check(A, k, f, pos, dtype, inter=False, **turn):  # noqa: F811
    """k [n, H, D] numbers of dtype, at positions pos [n]."""
    n, H, D = k.shape
    t = torch.from_numpy(np.asarray(k, np.float32)).to(DT[dtype]).cuda()[None]
    cache = A.kv4_cache(1, 1, H, n, D)
    one = torch.ones(1, n, 1, D, device="cuda", dtype=DT[dtype])
    weight = turn.pop("weight", None)
    w = None if weight is None else torch.from_numpy(weight.astype(np.float32)).cuda()
    r = A.kv4_append_rotated(cache, 0, one, t, torch.zeros_like(t), _i32([0]), f, positions=_i32(np.asarray(pos)[None]), k_weight=w, interleaved=inter, **turn)
    z = _z(_f64(t)[0], _f64(f), np.asarray(pos)[:, None], None if w is None else _f64(w), turn.get("eps"), inter, turn.get("scale", 1.0))
    back = A.kv4_read(cache, 0, _i32([0]), n, dtype=torch.float32)
    np.testing.assert_array_equal(_f64(back["k"])[0], O.held(z))
    want = np.where(np.isfinite(z).all((1, 2)), 0, A.ROW_NONFINITE)
    np.testing.assert_array_equal(r["status"].cpu().numpy()[0], want)
    return z


ROWS = pytest.mark.parametrize("dtype,D,inter", [(t, D, i) for t in ("f32", "bf16") for D in (64, 128) for i in (False, True)])


@ROWS
def test_numbers_beside_one_that_is_none(A, dtype, D, inter):  # noqa: F811
    """Next to borders between codes, which float32 could not decide."""
    rng = np.random.default_rng(D + inter)
    n, H = 400, 3
    k = torch.from_numpy(rng.standard_normal((n, H, D)).astype(np.float32)).to(DT[dtype]).double().numpy()
    f, pos = _freq(D), np.arange(n) * 37
    partner = np.arange(D) % 2 == 1 if inter else np.arange(D) >= D // 2
    bad = rng.integers(0, D, (n, H, 1))
    k[..., partner] = 0.0                                     # z_u = x_u cos, z_v = x_u sin
    z = _z(k, _f64(f), pos[:, None], inter=inter)
    step = _step(z)
    with np.errstate(all="ignore"):
        q = z / step
        near = np.floor(q) + 0.5
        near *= 1 + 2 * 2.0 ** -24 * (2 * rng.random(q.shape) - 1)
        # of the same groups only: the others have nothing that would decide the row again
        group = (np.arange(D) // (D // 8) == bad // (D // 8)) | (np.arange(D) // (D // 8) == (bad // (D // 8) if inter else (bad // (D // 8) + 4) % 8))
        k = np.where((np.abs(q) < 7) & (np.abs(q) > 0.3) & ~partner & group, k * near / q, k)
    np.put_along_axis(k, bad, rng.choice([np.nan, np.inf, -np.inf], bad.shape), -1)
    for turn in (dict(), dict(eps=1e-6)):
        z = _check(A, k, f, pos, dtype, inter, **turn)
        assert not np.isfinite(z).all((1, 2)).any()


@ROWS
def test_numbers_whose_turn_passes_float32(A, dtype, D, inter):  # noqa: F811
    """Pairs of 3e38 turned by any angle, alone and scaled, beside ordinary numbers: finite in 64 bits."""
    rng = np.random.default_rng(D + inter)
    n, H = 300, 3
    k = rng.standard_normal((n, H, D))
    j = rng.integers(0, D // 2, (n, H))
    for c in (2 * j, 2 * j + 1) if inter else (j, j + D // 2):
        np.put_along_axis(k, c[..., None], 3.3e38 * rng.choice([-1.0, 1.0], (n, H, 1)), -1)
    f, pos = _freq(D), rng.integers(0, 5000, n)
    pos[:20] = 0
    for turn in (dict(), dict(scale=1.3), dict(scale=2.0 ** 20), dict(scale=2.0 ** -20), dict(eps=1e-6), dict(eps=1e-6, scale=1.1)):
        z = _check(A, k, f, pos, dtype, inter, **turn)
        assert np.isfinite(z).all()
    # an angle that only the 64-bit sine has: a far partner's share of a small number
    tiny = torch.full((D // 2,), 2.0 ** -118, device="cuda")
    assert np.isfinite(_check(A, k, tiny, pos, dtype, inter, scale=1.3)).all()


@ROWS
def test_weights_of_any_size(A, dtype, D, inter):  # noqa: F811
    rng = np.random.default_rng(D + inter)
    n, H = 60, 40
    f, pos = _freq(D), rng.integers(0, 5000, n)
    w = rng.choice([-1.0, 1.0], (H, D)) * np.exp2(rng.uniform(-1, 1, (H, D)))
    w[:30] *= np.exp2(rng.integers(-120, 121, (30, 1)))        # a head's all
    w[5:20] *= np.exp2(rng.integers(-6, 7, (15, D)))
    for h in range(30, 36):                                    # one channel's
        w[h, rng.integers(0, D)] = [1e38, -1e38, 1e30, 1e-38, 0.0, 1e-45][h - 30]
    w = np.clip(w, -3e38, 3e38)
    for size in (1.0, 1e-3, 1e-18, 1e-37, 1e15, 1e24, 1e37):
        k = rng.standard_normal((n, H, D)) * size
        for eps in (1e-30, 1e-6):
            assert np.isfinite(_check(A, k, f, pos, dtype, inter, eps=eps, weight=w)).all()
    w[36, 3], w[37, D // 2], w[38, D - 1] = np.inf, -np.inf, np.nan
    z = _check(A, rng.standard_normal((n, H, D)), f, pos, dtype, inter, eps=1e-6, weight=w)
    assert not np.isfinite(z[:, 36:39]).all(-1).any() and np.isfinite(z[:, :36]).all()


@ROWS
def test_rows_of_all_sizes(A, dtype, D, inter):  # noqa: F811
    """Numbers of very different sizes in a row, normed and not."""
    rng = np.random.default_rng(D + inter)
    n, H = 200, 4
    k = rng.standard_normal((n, H, D)) * np.exp2(rng.integers(-100, 101, (n, H, 1)) + rng.integers(-20, 21, (n, H, D)))
    f, pos = _freq(D), rng.integers(0, 5000, n)
    for turn in (dict(), dict(scale=0.83), dict(eps=1e-30), dict(eps=1e-6), dict(eps=1.0, scale=1.2)):
        assert np.isfinite(_check(A, k, f, pos, dtype, inter, **turn)).all()


@ROWS
def test_scaled_numbers_on_borders(A, dtype, D, inter):  # noqa: F811
    """At position 0 a scale of a short decimal fraction makes products that 64 bits round onto a border between
    codes, or between steps, from a place that is not quite there."""
    rng = np.random.default_rng(D + inter)
    n, H = 300, 4
    k = rng.integers(-120, 121, (n, H, D)) * np.exp2(rng.integers(-8, 9, (n, H, 1)))
    for scale in (1.2, 1.3, 0.7, 1.1, 0.9, 5.2):
        _check(A, k, _freq(D), np.zeros(n, int), dtype, inter, scale=scale)
        _check(A, k, _freq(D // 2), np.zeros(n, int), dtype, inter, scale=scale)


@ROWS
def test_equal_numbers_under_slow_turns(A, dtype, D, inter):  # noqa: F811
    """Numbers of both signs that are equal but for what a turn of 2^-70 to 2^-30 adds: which of them is the
    largest, and so the step's sign, hangs on what 64 bits keep of it."""
    rng = np.random.default_rng(D + inter)
    n, H = 500, 4
    k = rng.choice([-1.0, 1.0], (n, H, D)) * rng.integers(5, 8, (n, H, D)) / 4
    f = torch.from_numpy((2.0 ** rng.uniform(-70, -30, D // 2)).astype(np.float32)).cuda()
    for turn in (dict(), dict(eps=1e-6), dict(scale=1.25), dict(scale=1.3)):
        _check(A, k, f, rng.integers(0, 50, n), dtype, inter, **turn)
