"""Host-side checks of the rotation calls: refusals before anything is launched, the
binding's checks, and the oracle against closed forms."""
import ctypes

import numpy as np
import pytest

from oracle import kv4 as K
from oracle import turn as O


class Turn(ctypes.Structure):  # aces_turn
    _fields_ = [("inv_freq", ctypes.c_void_p), ("rot_dim", ctypes.c_int), ("interleaved", ctypes.c_int), ("axes", ctypes.c_void_p),
                ("positions", ctypes.c_void_p), ("n_axes", ctypes.c_int), ("start", ctypes.c_void_p), ("base", ctypes.c_void_p),
                ("depth", ctypes.c_void_p), ("depth_stride", ctypes.c_int64), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("q_weight_dt", ctypes.c_int), ("k_weight_dt", ctypes.c_int), ("q_weight_stride", ctypes.c_int64),
                ("k_weight_stride", ctypes.c_int64), ("norm", ctypes.c_int), ("eps", ctypes.c_double), ("scale", ctypes.c_double)]


@pytest.fixture(scope="module")
def lib():
    from paper_2609_02514_gb300 import build
    import paper_2609_02514_gb300 as A
    build.build()
    return A.load()


FAKE = 0x10000   # never dereferenced: validation fails first


def _strides(n=3, heads=2, D=64):
    return (ctypes.c_int64 * 3)(n * heads * D, heads * D, D)


def _turn(start=True, **kw):
    t = dict(inv_freq=FAKE, rot_dim=64, n_axes=1, start=FAKE if start else None, scale=1.0)
    t.update(kw)
    return ctypes.byref(Turn(**t))


TURN_REFUSALS = [
    (dict(inv_freq=None), 1), (dict(rot_dim=0), 1), (dict(rot_dim=-16), 1), (dict(rot_dim=128), 1), (dict(rot_dim=24), 2), (dict(rot_dim=8), 2),
    (dict(positions=FAKE, n_axes=0), 1), (dict(positions=FAKE, n_axes=5, axes=FAKE), 1), (dict(positions=FAKE, n_axes=2), 1),
    (dict(depth=FAKE, depth_stride=2), 1), (dict(depth=FAKE, depth_stride=-3), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(scale=2.0 ** 21), 1), (dict(norm=1), 1), (dict(norm=1, eps=-1.0), 1),
    (dict(norm=1, eps=1e-31), 1), (dict(norm=1, eps=float("nan")), 1), (dict(norm=1, eps=1.5), 1), (dict(norm=1, eps=float("inf")), 1), (dict(q_weight=FAKE), 1),
    (dict(k_weight=FAKE), 1), (dict(norm=1, eps=1e-6, q_weight=FAKE, q_weight_dt=3), 2),
    (dict(norm=1, eps=1e-6, k_weight=FAKE, k_weight_stride=32), 1), (dict(norm=1, eps=1e-6, k_weight=FAKE + 2, k_weight_dt=0), 1)]


def _rotate(lib, turn=None, **kw):
    a = dict(q=FAKE, k=FAKE, dt=1, qs=_strides(heads=4), ks=_strides(), B=2, n=3, Hq=4, H=2, D=64, turn=turn or _turn(), qo=FAKE, ko=FAKE,
             qos=_strides(heads=4), kos=_strides(), s=None)
    a.update(kw)
    return lib.aces_rotate_qk(*a.values())


@pytest.mark.parametrize("kw,code", TURN_REFUSALS + [(dict(start=False), 1)])
def test_rotate_refuses_turns(lib, kw, code):
    assert _rotate(lib, _turn(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), 1), (dict(k=None), 1), (dict(q=FAKE + 1), 1), (dict(k=FAKE + 2, dt=0), 1), (dict(dt=7), 2), (dict(qs=None), 1), (dict(ks=None), 1),
    (dict(B=0), 1), (dict(n=0), 1), (dict(Hq=0), 1), (dict(H=0), 1), (dict(D=0), 1), (dict(D=96), 2), (dict(D=256), 2), (dict(qo=None), 1),
    (dict(ko=None), 1), (dict(qo=FAKE + 1), 1), (dict(qos=None), 1), (dict(kos=None), 1), (dict(n=1 << 30), 1), (dict(B=1 << 20, n=1 << 12), 1),
    # outputs whose numbers would share places
    (dict(qos=(ctypes.c_int64 * 3)(0, 256, 64)), 1), (dict(kos=(ctypes.c_int64 * 3)(384, 128, 32)), 1),
    (dict(qos=(ctypes.c_int64 * 3)(768, 128, 64)), 1)])
def test_rotate_refuses(lib, kw, code):
    assert _rotate(lib, **kw) == code


def test_rotate_refuses_no_turn(lib):
    a = [FAKE, FAKE, 1, _strides(heads=4), _strides(), 2, 3, 4, 2, 64, None, FAKE, FAKE, _strides(heads=4), _strides(), None]
    assert lib.aces_rotate_qk(*a) == 1


def _append(lib, turn=None, **kw):
    a = dict(cache=FAKE, planes=4, layer=1, B=2, H=2, S=64, D=64, q=FAKE, k=FAKE, v=FAKE, dt=1, qs=_strides(heads=4), ks=_strides(), vs=_strides(),
             Hq=4, start=FAKE, count=None, n=3, turn=turn or _turn(start=False), qo=FAKE, qos=_strides(heads=4), st=FAKE, s=None)
    a.update(kw)
    return lib.aces_kv4_append_rotated(*a.values())


@pytest.mark.parametrize("kw,code", TURN_REFUSALS)
def test_append_refuses_turns(lib, kw, code):
    assert _append(lib, _turn(**{"start": False, **kw})) == code


@pytest.mark.parametrize("kw,code", [
    (dict(cache=None), 1), (dict(cache=FAKE + 8), 1), (dict(planes=1), 1), (dict(layer=2), 1), (dict(layer=-1), 1), (dict(B=0), 1), (dict(H=0), 1),
    (dict(S=0), 1), (dict(D=0), 1), (dict(D=96), 2), (dict(dt=7), 2), (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(start=None), 1),
    (dict(n=0), 1), (dict(v=FAKE + 1), 1), (dict(qo=None), 1), (dict(qo=FAKE + 1), 1), (dict(st=None), 1), (dict(qs=None), 1), (dict(ks=None), 1),
    (dict(vs=None), 1), (dict(qos=None), 1), (dict(Hq=0), 1), (dict(turn=_turn()), 1), (dict(qos=(ctypes.c_int64 * 3)(768, 0, 64)), 1)])
def test_append_refuses(lib, kw, code):
    assert _append(lib, **kw) == code


def test_binding_refuses_host_tensors(lib):
    torch = pytest.importorskip("torch")
    import paper_2609_02514_gb300 as A
    x, f, at = torch.zeros(1, 1, 1, 64), torch.zeros(32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        A.rotate_qk(x, x, f, at)
    with pytest.raises(ValueError, match="CUDA"):
        A.kv4_append_rotated(torch.zeros(2, 1, 1, 8, 48, dtype=torch.uint8), 0, x, x, x, at, f)


# -- the oracle ---------------------------------------------------------------
def test_oracle_turns_by_hand():
    x = np.zeros((1, 2, 64))
    x[0, 0, 3], x[0, 1, 35] = 1.0, 2.0
    f = np.zeros(32)
    f[3] = np.pi / 2
    z, h = O.turned(x, f, np.array([[1]]))                   # a quarter: u becomes v, v becomes -u
    np.testing.assert_allclose(z[0, 0, [3, 35]], [0, 1], atol=1e-15)
    np.testing.assert_allclose(z[0, 1, [3, 35]], [-2, 0], atol=1e-15)
    assert h[0, 1, 3] == 2.0
    x = np.arange(64.0)[None, None]
    z, _ = O.turned(x, f, np.array([[2], [7]]), axes=np.where(np.arange(32) == 3, 0, 1), interleaved=True, scale=0.5)
    np.testing.assert_allclose(z[0, 0, 6:8], [-3.0, -3.5], atol=1e-14)      # half a turn
    np.testing.assert_allclose(z[0, 0, 8:], x[0, 0, 8:] / 2)


def test_oracle_keeps_lengths_and_differences():
    """A turn keeps a head's length, and products hang on the distance of positions only."""
    rng = np.random.default_rng(3)
    q, k = rng.standard_normal((2, 1, 128))
    f = 10000.0 ** (-np.arange(64) / 64)

    def at(x, p):
        return O.turned(x[None], f, np.array([[p]]))[0][0]
    np.testing.assert_allclose(np.linalg.norm(at(q, 12345)), np.linalg.norm(q))
    np.testing.assert_allclose((at(q, 40) * at(k, 7)).sum(), (at(q, 1040) * at(k, 1007)).sum())
    y, _ = O.turned(rng.standard_normal((1, 3, 64)) * 100, f[:8], np.array([[5]]), eps=1e-6)
    np.testing.assert_allclose((y ** 2).mean(-1), 1.0, rtol=1e-6)


def test_oracle_holds_what_the_caches_oracle_holds():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((40, 64)) * np.exp(3 * rng.standard_normal((40, 1)))
    x[3, 5], x[4], x[5, :8], x[6, 9] = np.nan, 0.0, [2, -2, 1, 1, 1, 1, 1, 1], 3e7
    np.testing.assert_array_equal(O.held(x), K.values_of(K.rows_of(x)))
