"""Tensors that a call writes for the caller say so to autograd: what was saved of them before is
not taken for the numbers that a gradient needs."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import A, _i32  # noqa: E402, F401
from tests.test_gpu_turn import _freq  # noqa: E402


def test_a_rotation_in_place_is_seen_by_autograd(A):  # noqa: F811
    x = torch.randn(2, 3, 4, 64, device="cuda", requires_grad=True)
    q = torch.sigmoid(x)                       # saves its result
    k = torch.randn(2, 3, 1, 64, device="cuda")
    A.rotate_qk(q, k, _freq(64), start=_i32([0, 5]), out=dict(q=q))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        q.sum().backward()


def test_versions_of_outputs(A):  # noqa: F811
    f, start = _freq(64), _i32([0])
    q, k = torch.randn(1, 2, 4, 64, device="cuda"), torch.randn(1, 2, 2, 64, device="cuda")
    cache = A.kv4_cache(1, 1, 2, 8, 64)
    made = A.kv4_append_rotated(cache, 0, q, k, k, start, f)
    made.update(A.kv4_shared_attention(q, cache, start, cache, 0, start))
    made = {key: t.clone() for key, t in made.items()}
    was = {key: t._version for key, t in made.items()}
    calls = [(("q", "k"), lambda o: A.rotate_qk(q, k, f, start=start, out=o)),
             (("out", "lse"), lambda o: A.kv4_attention(q, cache, 0, start, out=o)),
             (("out", "lse"), lambda o: A.kv4_shared_attention(q, cache, start, cache, 0, start, out=o)),
             (("q",), lambda o: A.kv4_append_rotated(cache, 0, q, k, k, start, f, out=o))]
    made["k"] = torch.empty_like(k)
    was["k"] = made["k"]._version
    for keys, call in calls:
        r = call({key: made[key] for key in keys})
        for key in keys:
            assert r[key] is made[key] and made[key]._version > was[key]
            was[key] = made[key]._version
    with torch.inference_mode():               # tensors that have no versions
        o = dict(q=torch.empty_like(q), k=torch.empty_like(k))
        r = A.rotate_qk(q, k, f, start=start, out=o)
    r = A.rotate_qk(q, k, f, start=start, out=o)
    assert r["q"] is o["q"] and torch.equal(r["q"], made["q"])
