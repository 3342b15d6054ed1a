"""Tensors on another GPU than the current one are refused: the library launches on
the current device.  (Host logic only: the current device is a stand-in.)"""
import pytest

torch = pytest.importorskip("torch")


def test_the_stream_is_the_current_devices(monkeypatch):
    import paper_2609_02514_gb300 as A
    asked = []
    monkeypatch.setattr(A, "_raw_stream", lambda i: asked.append(i) or 0)
    monkeypatch.setattr(A, "_current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:1.*cuda:0 is the current device"):
        A._stream(torch.device("cuda", 1))
    assert not asked
    assert A._stream(torch.device("cuda", 0)) == 0 and asked == [0]
    monkeypatch.setattr(A, "_current_device", lambda: 1)
    assert A._stream(torch.device("cuda", 1)) == 0 and asked == [0, 1]


@pytest.mark.gpu
def test_the_cache_calls_refuse_another_device(monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_02514_gb300 as A
    A.load()
    cache = A.kv4_cache(1, 1, 1, 8, 64)
    x = torch.ones(1, 1, 1, 64, device="cuda")
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    calls = [lambda: A.kv4_append(cache, 0, x, x, at), lambda: A.kv4_read(cache, 0, at, 1), lambda: A.kv4_attention(x, cache, 0, at)]
    for f in calls:
        f()
    torch.cuda.synchronize()
    before = cache.clone()
    monkeypatch.setattr(A, "_current_device", lambda: 1)     # as if another GPU were the current one
    x.fill_(2.0)
    for f in calls:
        with pytest.raises(ValueError, match="current device"):
            f()
    torch.cuda.synchronize()
    assert torch.equal(cache, before)
