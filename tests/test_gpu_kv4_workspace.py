"""kv4_attention's workspace: a call's own, given back behind it on the call's stream,
or the caller's."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_02514_gb300 as A
    A.load()
    return A


def _setting(A, n):
    B, Hq, H, D, S = 2, 8, 2, 128, 6000
    gen = torch.Generator(device="cuda").manual_seed(n)
    cache = A.kv4_cache(1, B, H, S, D)
    k, v = (torch.randn(B, S, H, D, generator=gen, device="cuda").bfloat16() for _ in range(2))
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    A.kv4_append(cache, 0, k, v, zero)
    q = torch.randn(B, n, Hq, D, generator=gen, device="cuda").bfloat16()
    P = torch.tensor([S - n, 3000], dtype=torch.int32, device="cuda")
    return q, cache, P


@pytest.mark.parametrize("n", [1, 3, 200])
def test_nothing_is_kept_for_a_stream(A, n):
    q, cache, P = _setting(A, n)
    want = A.kv4_attention(q, cache, 0, P)
    torch.cuda.synchronize()
    base = torch.cuda.memory_allocated()
    streams = [torch.cuda.Stream() for _ in range(6)]
    streams += [torch.cuda.ExternalStream(torch.cuda.Stream().cuda_stream)]
    for s in streams:
        with torch.cuda.stream(s):
            r = A.kv4_attention(q, cache, 0, P)
        s.synchronize()
        assert torch.equal(r["out"], want["out"]) and torch.equal(r["lse"], want["lse"])
        del r
    assert torch.cuda.memory_allocated() == base


def test_the_callers_workspace(A):
    q, cache, P = _setting(A, 40)
    need = A.kv4_workspace_bytes(2, 40, 8, 2, 128)
    want = A.kv4_attention(q, cache, 0, P)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    r = A.kv4_attention(q, cache, 0, P, workspace=ws[:need])
    torch.cuda.synchronize()
    assert torch.equal(r["out"], want["out"]) and (ws[need:] == 255).all()
    with pytest.raises(A.AcespecError):
        A.kv4_attention(q, cache, 0, P, workspace=ws[:need - 16])
    with pytest.raises(A.AcespecError):
        A.kv4_attention(q, cache, 0, P, workspace=ws[8:])
    for bad in (ws[::2], ws.cpu(), 7):
        with pytest.raises(ValueError):
            A.kv4_attention(q, cache, 0, P, workspace=bad)
