"""One token of so many heads that its steps times its slices pass 32 bits: the same bits as
as many tokens of one head at the same position."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import A  # noqa: E402, F401
from tests.test_gpu_turn import _freq, _i32  # noqa: E402


def test_a_token_of_millions_of_heads(A):  # noqa: F811
    N, D = 5_000_000, 64                       # 625 thousand steps of eight heads
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GB of device memory")
    q = torch.randn(1, 1, N, D, device="cuda", dtype=torch.bfloat16)
    k = torch.randn(1, 1, 3, D, device="cuda", dtype=torch.bfloat16)
    f = _freq(D)
    r = A.rotate_qk(q, k, f, start=_i32([77]), eps=1e-6)
    rows = q.view(1, N, 1, D)
    one = A.rotate_qk(rows, rows, f, positions=torch.full((1, N), 77, dtype=torch.int32, device="cuda"), eps=1e-6)
    assert torch.equal(r["q"].view(-1), one["q"].view(-1)) and torch.equal(one["q"], one["k"])
    last = A.rotate_qk(k, k, f, start=_i32([77]), eps=1e-6)
    assert torch.equal(r["k"], last["k"])
