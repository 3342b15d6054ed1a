"""The status of kv4_shared_attention's second pass when a wait gave up (which the checked build
is told to say; nothing waits): results that are not valid are not called so, whichever of a sequence's
CTAs comes last."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import _filled, _i32, _torch  # noqa: E402


@pytest.fixture
def A():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_02514_gb300 as A
    from paper_2609_02514_gb300 import build
    build.build(checked=True)
    A.use_checked(True)
    A.checked_shared_passes(2)
    yield A
    A.checked_late(-1)
    A.checked_shared_passes(0)
    A.use_checked(False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,S", [(3, 40), (3, 600), (100, 40), (3, 9000), (100, 9000)])   # a CTA an item, clusters, shares
@pytest.mark.parametrize("head", [0, 1, 3])
def test_a_wait_that_gave_up_is_in_the_status(A, dtype, B, S, head):
    H, D = 4, 64
    rng = np.random.default_rng(B)
    shared, _, _ = _filled(A, rng, 1, H, 50, D)
    cache = A.kv4_cache(1, B, H, S, D)
    q = _torch(rng.standard_normal((B, 1, 8, D)), dtype)
    P = rng.integers(0, S - 1, B)
    P[1] = S                                                  # its token is outside
    call = lambda: A.kv4_shared_attention(q, shared, _i32([50]), cache, 0, _i32(P))["status"].cpu().numpy()  # noqa: E731
    want = np.zeros(B, np.int32)
    want[1] = A.ROW_RANGE
    np.testing.assert_array_equal(call(), want)
    A.checked_late(head)
    r = call()
    A.checked_late(-1)
    assert (r & A.ROW_TIMEOUT)[want == 0].all() and ((r & ~A.ROW_TIMEOUT) == want).all()
    np.testing.assert_array_equal(call(), want)
