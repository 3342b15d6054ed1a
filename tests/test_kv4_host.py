"""Host-side checks of the 4-bit KV cache: refusals before anything is
launched, sizes, the binding's checks, and the oracle's format against closed
forms."""
import ctypes

import numpy as np
import pytest

from oracle import kv4 as O


@pytest.fixture(scope="module")
def lib():
    from paper_2609_02514_gb300 import build
    import paper_2609_02514_gb300 as A
    build.build()
    return A.load()


FAKE = ctypes.c_void_p(0x10000)   # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x10001)
ST = (ctypes.c_int64 * 3)(64, 64, 64)


def test_symbols_and_sizes(lib):
    for f in ("aces_kv4_row_bytes", "aces_kv4_append", "aces_kv4_read", "aces_kv4_workspace_bytes", "aces_kv4_attention"):
        assert hasattr(lib, f)
    assert [lib.aces_kv4_row_bytes(d) for d in (64, 128, 0, 96, 256)] == [48, 80, -1, -1, -1]
    ws = lib.aces_kv4_workspace_bytes
    assert ws(1, 1, 8, 2, 128) > 0
    for bad in ((0, 1, 8, 2, 128), (1, 0, 8, 2, 128), (1, 1, 8, 3, 128), (1, 1, 2, 4, 128), (1, 1, 8, 2, 96), (1 << 20, 1 << 12, 8, 2, 64)):
        assert ws(*bad) == 0, bad


def _append(lib, **kw):
    a = dict(cache=FAKE, planes=4, layer=1, B=2, H=2, S=64, D=64, k=FAKE, v=FAKE, dt=1, ks=ST, vs=ST, start=FAKE, count=None, n=3,
             st=FAKE, s=None)
    a.update(kw)
    return lib.aces_kv4_append(*a.values())


CACHE_REFUSALS = [(dict(cache=None), 1), (dict(cache=ctypes.c_void_p(0x10008)), 1), (dict(planes=1), 1), (dict(layer=2), 1), (dict(layer=-1), 1),
                  (dict(B=0), 1), (dict(H=0), 1), (dict(S=0), 1), (dict(D=0), 1), (dict(D=96), 2), (dict(dt=7), 2)]


@pytest.mark.parametrize("kw,code", CACHE_REFUSALS + [
    (dict(k=None), 1), (dict(v=None), 1), (dict(start=None), 1), (dict(st=None), 1), (dict(n=0), 1), (dict(ks=None), 1), (dict(vs=None), 1),
    (dict(k=ODD), 1), (dict(v=ctypes.c_void_p(0x10002), dt=0), 1)])
def test_append_refuses(lib, kw, code):
    assert _append(lib, **kw) == code


def _read(lib, **kw):
    a = dict(cache=FAKE, planes=4, layer=1, B=2, H=2, S=64, D=64, start=FAKE, n=3, k=FAKE, v=FAKE, dt=1, s=None)
    a.update(kw)
    return lib.aces_kv4_read(*a.values())


@pytest.mark.parametrize("kw,code", CACHE_REFUSALS + [
    (dict(k=None), 1), (dict(v=None), 1), (dict(start=None), 1), (dict(n=0), 1), (dict(k=ctypes.c_void_p(0x10008)), 1)])
def test_read_refuses(lib, kw, code):
    assert _read(lib, **kw) == code


def _attend(lib, **kw):
    a = dict(q=FAKE, dt=1, qs=ST, cache=FAKE, planes=4, layer=1, B=2, n=3, Hq=4, H=2, S=64, D=64, P=FAKE, count=None, mask=None, ms=0,
             depth=None, ds=0, scale=0.1, window=0, sinks=0, out=FAKE, lse=None, st=FAKE, ws=FAKE, wsb=1 << 40, s=None)
    a.update(kw)
    return lib.aces_kv4_attention(*a.values())


@pytest.mark.parametrize("kw,code", CACHE_REFUSALS + [
    (dict(q=None), 1), (dict(qs=None), 1), (dict(P=None), 1), (dict(out=None), 1), (dict(st=None), 1), (dict(ws=None), 1), (dict(n=0), 1),
    (dict(Hq=3), 1), (dict(Hq=1), 1), (dict(q=ODD), 1), (dict(out=ctypes.c_void_p(0x10008)), 1), (dict(ws=ctypes.c_void_p(0x10008)), 1),
    (dict(wsb=0), 1), (dict(mask=FAKE), 1), (dict(depth=FAKE), 1), (dict(mask=FAKE, depth=FAKE, ms=2), 1),
    (dict(mask=FAKE, depth=FAKE, ds=2), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(window=-1), 1), (dict(sinks=-1), 1)])
def test_attention_refuses(lib, kw, code):
    assert _attend(lib, **kw) == code


def test_binding_refuses_host_tensors(lib):
    torch = pytest.importorskip("torch")
    import paper_2609_02514_gb300 as A
    cache = torch.zeros(2, 1, 1, 8, 48, dtype=torch.uint8)
    x = torch.zeros(1, 1, 1, 64)
    with pytest.raises(ValueError):
        A.kv4_append(cache, 0, x, x, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        A.kv4_read(cache, 0, torch.zeros(1, dtype=torch.int32), 1)
    with pytest.raises(ValueError):
        A.kv4_attention(x, cache, 0, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        A.kv4_cache(1, 1, 1, 8, 96, device="cpu")
    assert tuple(A.kv4_cache(3, 2, 4, 8, 128, device="cpu").shape) == (6, 2, 4, 8, 80)


# -- the oracle's format ------------------------------------------------------
def test_oracle_rows_by_hand():
    x = np.zeros(64)
    x[0:8] = [8, -8, 1, 2, 3, 4, 5, 7.6]      # a = 8: the step is -1, 8 lies on -8, -8 clamps to 7
    row = O.row_of(x)
    codes = [0, 15, 7, 6, 5, 4, 3, 0]          # 8 - x, ties to even (7.6 -> -8)
    word = 0
    for e, c in enumerate(codes):
        word |= c << (4 * (e // 2) + 16 * (e % 2))
    assert int(row[:4].view(np.uint32)[0]) == word
    assert [int(w) for w in row[4:32].view(np.uint32)] == [0x88888888] * 7
    t = (row[32:].view(np.uint16).astype(np.uint32) << 16).view(np.float32)
    assert t[0] == -(2.0 ** -16) and not t[1:].any()
    assert list(O.values_of(row[None])[0, :8]) == [8, -7, 1, 2, 3, 4, 5, 8]


def test_oracle_values_survive_a_second_writing():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((20, 128)) * 100
    once = O.values_of(O.rows_of(x))
    step = np.abs([[O.step_of(r[g * 16:g * 16 + 16]) for g in range(8)] for r in x])
    off = np.abs(once - x).reshape(20, 8, 16)
    assert (off <= 1.25 * step[..., None]).all() and np.mean(off <= 0.5 * step[..., None]) > 0.97
    twice = O.values_of(O.rows_of(once))
    same = np.abs(twice - once).reshape(20, 8, 16).max(-1) == 0       # all groups whose largest lies on -8
    assert same.mean() > 0.9


def test_oracle_attention_pins():
    """Equal scores give the mean, one key its value, and lse its score."""
    rng = np.random.default_rng(2)
    V = rng.standard_normal((5, 64))
    q = rng.standard_normal((2, 64))
    out, lse, _, _ = O.attend(q * 0, V, V, np.ones((2, 5), bool), 0.3)
    np.testing.assert_allclose(out, np.broadcast_to(V.mean(0), (2, 64)), rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(lse, np.log(5.0))
    ok = np.array([[False, True, False, False, False], [False] * 5])
    out, lse, _, _ = O.attend(q, V, V, ok, 0.3)
    np.testing.assert_allclose(out[0], V[1])
    np.testing.assert_allclose(lse[0], 0.3 * q[0] @ V[1])
    assert not out[1].any() and np.isneginf(lse[1])
    ok = O.visible(3, 2, 2, 6, window=2, sinks=1)
    np.testing.assert_array_equal(ok, [[1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0]])
