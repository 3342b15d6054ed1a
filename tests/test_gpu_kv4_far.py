"""Attention whose keys and values lie past 2^32 bytes of a plane, in the second layer:
results and lse against float64, through each kernel (clusters, shares and a join, the
tensor-core kernel).  What is seen lies behind a window, so the reference needs the
last positions only.  Bounds as in test_gpu_kv4.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import A, _compare, _f64, _i32, _torch  # noqa: E402, F401

B, H, Hq, D, S, N, BACK = 65, 1, 2, 128, 830000, 40, 4100


@pytest.fixture(scope="module")
def far(A):  # noqa: F811
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    cache = torch.empty(4, B, H, S, D // 2 + 16, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(9)
    at = S - N - 1                                           # the last sequence's prefix
    assert ((B - 1) * S + at - BACK) * (D // 2 + 16) > 1 << 32
    start = _i32([0] * (B - 1) + [at - BACK])
    k, v = (torch.randn(B, BACK + N, H, D, generator=gen, device="cuda") for _ in range(2))
    k *= torch.exp(0.5 * torch.randn(B, BACK + N, H, 1, generator=gen, device="cuda"))
    A.kv4_append(cache, 1, k, v, start)
    back = A.kv4_read(cache, 1, start, BACK + N, dtype=torch.float32)
    K, V = (_f64(back[x][B - 1:]).swapaxes(1, 2) for x in ("k", "v"))
    prefix = _i32([0] * (B - 1) + [at])
    yield cache, K, V, prefix
    del cache
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,window", [(1, 1), (1, 64), (1, 4000), (7, 300), (7, 4000), (N, N), (N, 500), (N, 4000)])
def test_far_keys_and_values(A, far, n, window, dtype):  # noqa: F811
    cache, K, V, prefix = far
    rng = np.random.default_rng(n + window)
    q = _torch(rng.standard_normal((B, n, Hq, D)), dtype)
    r = A.kv4_attention(q, cache, 1, prefix, window=window)
    assert not r["status"].any()
    # positions counted from BACK before the prefix: the window ends what lies before
    last = {x: r[x][B - 1:] for x in ("out", "lse")}
    _compare(last, _f64(q[B - 1:]), K[:, :, :BACK + n], V[:, :, :BACK + n], [BACK], [n], dtype, D ** -0.5, window=window)
