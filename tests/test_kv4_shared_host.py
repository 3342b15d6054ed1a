"""Host-side checks of the attention behind shared prefixes: refusals before anything is
launched, sizes, the binding's checks."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2609_02514_gb300 import build
    import paper_2609_02514_gb300 as A
    build.build()
    return A.load()


FAKE = ctypes.c_void_p(0x10000)   # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x10001)
OFF = ctypes.c_void_p(0x10008)
ST = (ctypes.c_int64 * 3)(64, 64, 64)


def test_sizes(lib):
    ws, own = lib.aces_kv4_shared_workspace_bytes, lib.aces_kv4_workspace_bytes
    assert ws(4, 1, 3, 8, 2, 128) >= 4 * 3 * 8 * (128 + 2) * 4 + own(4, 3, 8, 2, 128)
    assert ws(4, 2, 3, 8, 2, 64) % 16 == 0
    for bad in ((0, 1, 1, 8, 2, 128), (4, 0, 1, 8, 2, 128), (4, 3, 1, 8, 2, 128), (2, 4, 1, 8, 2, 128), (4, 1, 0, 8, 2, 128), (4, 1, 1, 8, 3, 128),
                (4, 1, 1, 8, 2, 96), (1 << 20, 1, 1 << 12, 8, 2, 64)):
        assert ws(*bad) == 0, bad


def _attend(lib, **kw):
    a = dict(q=FAKE, dt=1, qs=ST, shared=FAKE, sp=4, groups=2, S0=32, sl=FAKE, cache=FAKE, planes=4, layer=1, B=4, n=3, Hq=4, H=2, S=64, D=64,
             P=FAKE, count=None, mask=None, ms=0, depth=None, ds=0, scale=0.1, window=0, sinks=0, out=FAKE, lse=None, st=FAKE, ws=FAKE,
             wsb=1 << 40, s=None)
    a.update(kw)
    return lib.aces_kv4_shared_attention(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(cache=None), 1), (dict(cache=OFF), 1), (dict(planes=1), 1), (dict(layer=2), 1), (dict(layer=-1), 1), (dict(B=0), 1), (dict(H=0), 1),
    (dict(S=0), 1), (dict(D=0), 1), (dict(D=96), 2), (dict(dt=7), 2), (dict(shared=None), 1), (dict(shared=OFF), 1), (dict(sp=1), 1), (dict(sp=2), 1),
    (dict(groups=0), 1), (dict(groups=3), 1), (dict(groups=8), 1), (dict(groups=-1), 1), (dict(S0=0), 1), (dict(sl=None), 1), (dict(q=None), 1),
    (dict(qs=None), 1), (dict(P=None), 1), (dict(out=None), 1), (dict(st=None), 1), (dict(ws=None), 1), (dict(n=0), 1), (dict(Hq=3), 1),
    (dict(Hq=1), 1), (dict(q=ODD), 1), (dict(out=OFF), 1), (dict(ws=OFF), 1), (dict(wsb=0), 1), (dict(wsb=4 * 3 * 4 * 66 * 4), 1), (dict(mask=FAKE), 1),
    (dict(depth=FAKE), 1), (dict(mask=FAKE, depth=FAKE, ms=2), 1), (dict(mask=FAKE, depth=FAKE, ds=2), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(window=-1), 1), (dict(sinks=-1), 1)])
def test_attention_refuses(lib, kw, code):
    assert _attend(lib, **kw) == code


def test_binding_refuses_host_tensors(lib):
    torch = pytest.importorskip("torch")
    import paper_2609_02514_gb300 as A
    cache = torch.zeros(2, 1, 1, 8, 48, dtype=torch.uint8)
    at = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        A.kv4_shared_attention(torch.zeros(1, 1, 1, 64), cache, at, cache, 0, at)
