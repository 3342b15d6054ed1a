"""The 4-bit cache's calls when memory is short: torch's own out-of-memory error, and
nothing of the call left behind.  The limit is torch's allocator's own, for this
process."""
import contextlib

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


@contextlib.contextmanager
def _room_for(nbytes):
    """Lets torch reserve that much more than it has allocated."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    total = torch.cuda.get_device_properties(0).total_memory
    torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + nbytes) / total)
    try:
        yield
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)


MB = 1 << 20


def test_a_read_without_room_for_the_values(A):
    cache = A.kv4_cache(1, 1, 1, 64, 128)
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    n = 1 << 20                                              # 512 MB each in float32
    base = torch.cuda.memory_allocated()
    with _room_for(800 * MB):
        with pytest.raises(torch.OutOfMemoryError):
            A.kv4_read(cache, 0, at, n, dtype=torch.float32)
        assert torch.cuda.memory_allocated() == base
    back = A.kv4_read(cache, 0, at, 64)
    assert not back["k"].any()


def test_an_attention_without_room_for_its_lse(A):
    n, Hq, H, D = 1 << 17, 32, 4, 128                        # out 1 GB, lse 16 MB, workspace 41 MB
    cache = A.kv4_cache(1, 1, H, 64, D)
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.ones(1, 1, 1, D, dtype=torch.bfloat16, device="cuda").expand(1, n, Hq, D)
    base = torch.cuda.memory_allocated()
    with _room_for(1024 * MB + 50 * MB):
        with pytest.raises(torch.OutOfMemoryError):
            A.kv4_attention(q, cache, 0, at)
        assert torch.cuda.memory_allocated() == base
