"""kv4_shared_attention in one pass and in two, each asked for by name of the checked build, for
every shape, mask, window and status of test_gpu_kv4_shared.py and for windows with masks and first
tokens that reach from the prefix into a sequence's own rows; and the product library at sizes for
which its rule takes two.  Bounds are those of the tests that are called."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import tests.test_gpu_far_shared as FAR  # noqa: E402
import tests.test_gpu_kv4_shared as T  # noqa: E402
import tests.test_gpu_shared_cycle as C  # noqa: E402
from tests.test_gpu_far_shared import far  # noqa: E402, F401
from tests.test_gpu_kv4 import _f64, _filled, _i32, _torch, _tree_bits, _words  # noqa: E402


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_02514_gb300 as A
    from paper_2609_02514_gb300 import build
    build.build(checked=True)
    A.use_checked(True)
    A.checked_violation()
    yield A
    A.use_checked(False)


@pytest.fixture(params=[1, 2])
def passes(A, request):
    """As many passes, in every call of the test."""
    A.checked_shared_passes(request.param)
    yield request.param
    taken = A.checked_shared_passes(0)
    assert A.checked_violation() is None and taken == request.param


# B, n, Hq, H, D, prefixes' positions, own positions, form, window, sinks (n of trees: the form's)
MORE = [
    (3, 0, 8, 2, 128, [90], [50, 0, 7], "tree", 40, 3),                     # windows that end in the prefix, few rows
    (3, 0, 4, 2, 64, [9], [50, 0, 7], "tree", 12, 14),                      # first tokens beyond the prefix
    (4, 0, 4, 4, 64, [9, 300], [3, 11, 60, 0], "tree", 2, 20),
    (2, 0, 16, 2, 128, [20], [129, 3], "bigtree", 30, 33),                  # the same, many rows
    (2, 0, 16, 2, 64, [500], [40, 3], "bigtree", 300, 2),
    (4, 0, 16, 2, 128, [5, 140], [200, 0, 131, 9], "bigtree", 64, 150),
    (3, 41, 6, 2, 64, [20, 5, 0], [60, 300, 5], "causal", 40, 30),
    (2, 200, 4, 2, 128, [70], [150, 0], "causal", 130, 100),
    (40, 1, 8, 2, 128, [50], [2 * b for b in range(40)], "causal", 30, 70),
    (2, 150, 4, 4, 64, [129], [300, 257], "causal", 100, 5),                # windows shorter than the own rows
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", T.SHAPES + MORE, ids=lambda c: "-".join(map(str, c)).replace(" ", "")[:60])
def test_every_shape(A, passes, case, dtype):
    T.test_attention_is_the_definition(A, case, dtype, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,H", [(6, 4, 2), (50, 6, 2)])
def test_any_mask_any_strides(A, passes, dtype, n, Hq, H):
    T.test_any_mask_any_strides(A, dtype, n, Hq, H, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40])
def test_status_and_bad_queries(A, passes, dtype, n):
    T.test_sequences_outside_the_caches(A, dtype, n, 1)
    T.test_a_bad_query_spoils_its_own_row(A, n, dtype, 1)


@pytest.mark.parametrize("n,B", [(1, 3), (1, 50), (40, 3)])
def test_it_is_the_attention_over_one_cache(A, passes, n, B):
    T.test_it_is_the_attention_over_one_cache(A, n, B, 1)


def test_graphs_streams_and_workspaces(A, passes):
    T.test_graphs_streams_and_workspaces(A, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("per,n,window", [(1, 1, 4000), (2, 1, 64), (20, 1, 4000), (1, 40, 500), (2, 40, 4000)])
def test_far_prefixes(A, passes, far, per, n, window, dtype):  # noqa: F811
    FAR.test_far_prefixes(A, far, per, n, window, dtype)


@pytest.mark.parametrize("sizes", [dict(), dict(B=20, system=700, Hq=12, H=4, D=128, F=(3, 2, 1), branch_len=1)])
def test_the_calls_together(A, passes, sizes):
    spec = importlib.util.spec_from_file_location("edge_shared", os.path.join(C.ROOT, "examples", "edge_shared.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    C.test_a_cache_each_holds_the_same_rows(example, sizes)


# B, groups, n (0: a tree), Hq, H, D, dtype, the prefixes' room, window, sinks
@pytest.mark.parametrize("B,groups,n,Hq,H,D,dtype,room,window,sinks", [
    (64, 1, 1, 32, 8, 128, "bf16", 16384, 0, 0), (64, 2, 1, 12, 4, 64, "f32", 60000, 0, 0), (128, 1, 1, 8, 8, 64, "bf16", 9000, 1200, 4),
    (32, 2, 0, 32, 8, 128, "bf16", 20000, 0, 0), (48, 1, 0, 16, 8, 64, "bf16", 9000, 8000, 2000), (96, 1, 3, 4, 4, 64, "f32", 5000, 4000, 1600)])
def test_the_rule_takes_two(A, B, groups, n, Hq, H, D, dtype, room, window, sinks):
    rng = np.random.default_rng(B + D)
    mask = depth = words = dev_depth = None
    if n == 0:
        mask, depth = _tree_bits([3] * 8, 1)
        n, words, dev_depth = len(depth), _words(mask), _i32(depth)
    lens = [1500 - 90 * g for g in range(groups)]
    P, cnt = [int(x) for x in rng.integers(0, 60, B)], [n] * B
    shared, K0, V0 = _filled(A, rng, groups, H, max(lens), D)
    wide = torch.full((2, groups, H, room, D // 2 + 16), 255, dtype=torch.uint8, device="cuda")
    wide[:, :, :, :max(lens)] = shared
    cache, K, V = _filled(A, rng, B, H, 60 + n, D)
    q = _torch(rng.standard_normal((B, n, Hq, D)), dtype)
    call = lambda: A.kv4_shared_attention(q, wide, _i32(lens), cache, 0, _i32(P), mask=words, depth=dev_depth, window=window, sinks=sinks)  # noqa: E731
    A.checked_shared_passes(0)
    checked = call()
    assert A.checked_shared_passes(0) == 2 and A.checked_violation() is None
    A.use_checked(False)
    try:
        r = call()
        torch.cuda.synchronize()
    finally:
        A.use_checked(True)
    assert torch.equal(r["out"], checked["out"]) and torch.equal(r["lse"], checked["lse"]) and not r["status"].any()
    for b in (0, 1, B // 2 - 1, B // 2, B - 1):
        g = b // (B // groups)
        T._check({key: r[key][b:b + 1] for key in ("out", "lse")}, _f64(q)[b:b + 1], (K0[g:g + 1], V0[g:g + 1]), lens[g:g + 1],
                 (K[b:b + 1], V[b:b + 1]), P[b:b + 1], cnt[b:b + 1], dtype, D ** -0.5, mask, depth, window, sinks)


@pytest.mark.parametrize("B", [64, 95, 96, 97, 160])
def test_the_order_of_sequences(A, B):
    """In more than one wave, longest first up to 96: of all lengths, equal ones, and some outside the cache."""
    Hq, H, D, S = 8, 8, 64, 1040
    rng = np.random.default_rng(B)
    shared, K0, V0 = _filled(A, rng, 1, H, 50, D)
    cache, K, V = _filled(A, rng, B, H, S, D)
    P = rng.integers(0, S, B)
    P[::7], P[5], P[B // 2] = 900, S, -1
    q = _torch(rng.standard_normal((B, 1, Hq, D)), "bf16")
    A.checked_shared_passes(2)
    r = A.kv4_shared_attention(q, shared, _i32([50]), cache, 0, _i32(P))
    assert A.checked_shared_passes(0) == 2 and A.checked_violation() is None
    inside = (P >= 0) & (P < S)
    np.testing.assert_array_equal(r["status"].cpu().numpy(), np.where(inside, 0, A.ROW_RANGE))
    assert not r["out"][torch.from_numpy(~inside).cuda()].any()
    for b in np.flatnonzero(inside):
        T._check({key: r[key][b:b + 1] for key in ("out", "lse")}, _f64(q)[b:b + 1], (K0, V0), [50], (K[b:b + 1], V[b:b + 1]), [int(P[b])], [1], "bf16", D ** -0.5)
