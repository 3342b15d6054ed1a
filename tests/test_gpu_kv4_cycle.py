"""The edge's cycle over a 4-bit cache (examples/edge_kv4.py), and the kernels of
the cache in the checked build, whose record of indices out of range stays empty."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import kv4 as O  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("edge_kv4", os.path.join(ROOT, "examples", "edge_kv4.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.fixture(params=["product", "checked"])
def A(request):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_02514_gb300 as A
    if request.param == "checked":
        from paper_2609_02514_gb300 import build
        build.build(checked=True)
        A.use_checked(True)
        A.checked_violation()
    yield A
    if request.param == "checked":
        assert A.checked_violation() is None
        A.use_checked(False)


def test_cycle_ends_with_the_accepted_tokens_rows(A, example):
    """After the cycle the cache holds the prompt, the accepted tokens and the hit
    branch: the rows the tree had for them, moved and not rewritten."""
    F, L, K, prompt, n = (3, 2, 1, 1), 2, 4, 300, 4 + 7 * 2
    kinds = set()
    for seed in range(6):
        r = example.cycle(seed=seed)
        torch.cuda.synchronize()
        assert torch.isfinite(r["hidden"]).all()
        al, slot, new = (r[k].tolist() for k in ("accept_len", "slot", "new_len"))
        for b in range(len(al)):
            kinds.add(0 if slot[b] >= 0 else slot[b])
            assert new[b] == prompt + (al[b] + L if slot[b] >= 0 else K if slot[b] == -2 else al[b])
    assert len(kinds) >= 2


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_cycle_is_the_float64_one(A, example, window, sinks):
    """The last token's first layer over the moved cache, in float64 from the
    cache's own numbers."""
    B, Hq, H, D = 4, 8, 2, 64
    r = example.cycle(seed=11, window=window, sinks=sinks)
    gen = torch.Generator(device="cuda").manual_seed(5)
    q = torch.randn(B, 1, Hq, D, generator=gen, device="cuda").bfloat16()
    S = r["cache"].shape[3]
    got = A.kv4_attention(q, r["cache"], 0, r["new_len"], window=window, sinks=sinks)
    kv = O.values_of(r["cache"][:2].cpu().numpy())
    q64 = q.double().cpu().numpy()
    for b in range(B):
        P = int(r["new_len"][b])
        ok = O.visible(P, 1, 1, S, window=window, sinks=sinks)
        for hq in range(Hq):
            w, z, mag, M = O.attend(q64[b, :, hq], kv[0, b, hq // 4], kv[1, b, hq // 4], ok, D ** -0.5)
            # the two roundings of bfloat16 weights and results, as in test_gpu_kv4.py
            off = np.abs(got["out"][b, :, hq].double().cpu().numpy() - w)
            assert (off <= (2.0 ** -7 + 2.0 ** -17 + 2.0 ** -18 * (M[0] + 1)) * mag).all()


@pytest.mark.parametrize("n,Hq,H,D,P", [(1, 8, 2, 128, [0, 77, 700]), (3, 12, 4, 64, [5, 0, 300]), (1, 4, 4, 64, [5000, 3, 60]),
                                        (40, 8, 2, 128, [0, 129, 500]), (70, 4, 1, 64, [300, 1, 0]), (300, 2, 2, 64, [9, 0, 140])])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_kernels_stay_inside(A, n, Hq, H, D, P, dtype):
    """Ragged shapes whose last positions are the cache's last (the checked build
    looks at every index)."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    B, S = 3, max(P) + n
    cache = A.kv4_cache(2, B, H, S, D)
    start = torch.tensor(P, dtype=torch.int32, device="cuda")
    k, v = (torch.randn(B, S, H, D, generator=gen, device="cuda").to(dtype) for _ in range(2))
    A.kv4_append(cache, 1, k, v, torch.zeros_like(start))
    q = torch.randn(B, n, Hq, D, generator=gen, device="cuda").to(dtype)
    for window, sinks in ((0, 0), (50, 3)):
        r = A.kv4_attention(q, cache, 1, start, window=window, sinks=sinks)
        torch.cuda.synchronize()
        assert torch.isfinite(r["out"]).all() and not r["status"].any()
    bad = torch.tensor([S - n + 1, -3, 1 << 30], dtype=torch.int32, device="cuda")
    st = A.kv4_append(cache, 0, k[:, :n].contiguous(), v[:, :n].contiguous(), bad)
    r = A.kv4_attention(q, cache, 1, bad)
    back = A.kv4_read(cache, 1, bad, n, dtype=dtype)
    torch.cuda.synchronize()
    assert (r["status"] == A.ROW_RANGE).all() and not r["out"].any() and st[2].eq(A.ROW_RANGE).all() and not back["k"][2].any()
