"""kv4_shared_attention against float64 numpy over each sequence's rows in one piece: its
prefix's, then its own.  Short prefixes are read by every sequence; a pass of their own goes
by the shared cache's capacity, so the same sizes run both ways.  The bounds are test_gpu_kv4.py's; the two passes' sums come
together as its pieces do (an exponential, a product and an add each in float32, 2^-21
together), which its 2^-17 for exponentials and sums has room for."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_kv4 import _compare, _f64, _filled, _i32, _torch, _tree_bits, _words  # noqa: E402


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
    else:
        A.load()
    yield A
    if request.param == "checked":
        assert A.checked_violation() is None
        A.use_checked(False)


def _check(r, q, shared, lens, own, P, cnt, dtype, scale, mask=None, depth=None, window=0, sinks=0):
    """shared, own: (K, V) of [groups, H, S0, D] and [B, H, S, D]."""
    B = q.shape[0]
    per = B // len(lens)
    for b in range(B):
        g = b // per
        K, V = (np.concatenate([s[g, :, :lens[g]], o[b]], 1)[None] for s, o in zip(shared, own))
        m = mask[b] if mask is not None and mask.ndim == 3 else mask
        d = depth[b] if depth is not None and depth.ndim == 2 else depth
        _compare({key: r[key][b:b + 1] for key in ("out", "lse")}, q[b:b + 1], K, V, [lens[g] + P[b]], [cnt[b]], dtype, scale, m, d, window, sinks)


# B, n, Hq, H, D, prefixes' positions, own positions, form, window, sinks
SHAPES = [
    (1, 1, 1, 1, 64, [1], [0], "causal", 0, 0),                              # the least
    (3, 1, 8, 2, 128, [33], [0, 5, 31], "causal", 0, 0),                     # few rows in both passes
    (2, 1, 4, 4, 128, [2000], [700, 3], "causal", 0, 0),                     # clusters
    (4, 1, 12, 4, 64, [300, 0], [1, 40, 0, 9], "causal", 0, 0),              # two prefixes, one empty
    (40, 1, 8, 2, 128, [700], list(range(40)), "causal", 0, 0),              # 160 rows of the prefix: tensor cores, two halves of a tile
    (20, 1, 4, 2, 64, [129], [7] * 20, "causal", 0, 0),                      # 40 rows: one half
    (66, 1, 16, 2, 64, [257, 60, 128], [2] * 66, "causal", 0, 0),            # rows that cross tiles, three prefixes
    (9, 2, 8, 1, 128, [515], [100, 0, 3] * 3, "causal", 0, 0),
    (2, 70, 4, 2, 128, [200], [130, 1], "causal", 0, 0),                     # many rows in both
    (3, 41, 6, 2, 64, [100, 90, 0], [0, 300, 5], "causal", 0, 0),
    (2, 300, 2, 2, 64, [640], [0, 129], "causal", 0, 0),
    (3, 0, 8, 2, 128, [400], [50, 0, 7], "tree", 0, 0),
    (2, 0, 16, 2, 128, [130], [129, 3], "bigtree", 0, 0),
    (4, 1, 8, 2, 128, [900], [0, 40, 99, 101], "causal", 100, 4),            # windows that leave the prefix, or not
    (4, 1, 4, 4, 64, [2, 0], [10, 0, 50, 3], "causal", 8, 5),                # first tokens in the prefix and in the own rows
    (36, 1, 8, 2, 64, [700], [3 * b for b in range(36)], "causal", 64, 3),
    (3, 50, 4, 2, 64, [333], [0, 20, 90], "causal", 64, 70),
    (2, 0, 4, 2, 128, [60], [9, 0], "tree", 5, 2),
    (2, 0, 16, 2, 64, [200], [1, 60], "bigtree", 30, 130),
]


def _roomy(A, shared):
    """The same prefixes in a cache of 3 million positions (of all of them together)."""
    planes, groups, H, S0, R = shared.shape
    wide = torch.empty(planes, groups, H, 3_000_000 // (groups * H), R, dtype=torch.uint8, device="cuda")
    wide[:, :, :, :S0] = shared
    wide[:, :, :, S0:S0 + 200] = 255
    return wide


@pytest.mark.parametrize("passes", [1, 2])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "-".join(map(str, c)).replace(" ", "")[:60])
def test_attention_is_the_definition(A, case, dtype, passes):
    B, n, Hq, H, D, lens, P, form, window, sinks = case
    rng = np.random.default_rng(B + 7 * n + Hq + lens[0])
    mask = depth = words = dev_depth = None
    if form != "causal":
        mask, depth = _tree_bits([2, 1, 2], 2) if form == "tree" else _tree_bits([4] * 8, 1)
        n = len(depth)
        words, dev_depth = _words(mask), _i32(depth)
    cnt = [max(0, n - 3 * (b % 2)) for b in range(B)]
    S0, S = max(max(lens) + 2, 1), max(P) + n + 3
    shared, K0, V0 = _filled(A, rng, len(lens), H, S0, D, layers=2, layer=1)
    cache, K, V = _filled(A, rng, B, H, S, D, layers=3, layer=1)
    for g, m in enumerate(lens):
        shared[:, g, :, m:] = 255                               # bytes nobody wrote
    for b in range(B):
        cache[:, b, :, P[b] + cnt[b]:] = 255
    q = _torch(rng.standard_normal((B, n, Hq, D)) * 0.8, dtype)
    if passes == 2:
        shared = _roomy(A, shared)
    r = A.kv4_shared_attention(q, shared, _i32(lens), cache, 1, _i32(P), mask=words, depth=dev_depth, count=_i32(cnt), window=window,
                               sinks=sinks)
    torch.cuda.synchronize()
    assert not r["status"].any()
    _check(r, _f64(q), (K0, V0), lens, (K, V), P, cnt, dtype, D ** -0.5, mask, depth, window, sinks)


# windows so wide, of so many sequences, that the prefix has its own pass
@pytest.mark.parametrize("B,groups,n,Hq,H,D,length,window,sinks,dtype", [
    (128, 1, 1, 8, 8, 64, 1500, 1000, 4, "bf16"), (96, 2, 1, 16, 8, 128, 1300, 1200, 1300, "bf16"), (128, 1, 1, 4, 4, 64, 1100, 700, 7, "f32"),
    (24, 1, 20, 16, 8, 64, 6500, 6000, 5, "bf16")])
def test_windows_of_large_batches(A, B, groups, n, Hq, H, D, length, window, sinks, dtype):
    rng = np.random.default_rng(B)
    lens = [length - 100 * g for g in range(groups)]
    shared, K0, V0 = _filled(A, rng, groups, H, length + 900, D)
    cache, K, V = _filled(A, rng, B, H, 60 + n, D)
    P, cnt = [int(x) for x in rng.integers(0, 60, B)], [n] * B
    q = _torch(rng.standard_normal((B, n, Hq, D)), dtype)
    r = A.kv4_shared_attention(q, shared, _i32(lens), cache, 0, _i32(P), window=window, sinks=sinks)
    for b in (0, 1, B // 2 - 1, B // 2, B - 1):
        g = b // (B // groups)
        _check({key: r[key][b:b + 1] for key in ("out", "lse")}, _f64(q)[b:b + 1], (K0[g:g + 1], V0[g:g + 1]), lens[g:g + 1], (K[b:b + 1], V[b:b + 1]),
               P[b:b + 1], cnt[b:b + 1], dtype, D ** -0.5, window=window, sinks=sinks)


@pytest.mark.parametrize("passes", [1, 2])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,H", [(6, 4, 2), (50, 6, 2)])
def test_any_mask_any_strides(A, dtype, n, Hq, H, passes):
    """A mask and depths of every sequence, rows that see nothing, another scale, and
    queries inside a wider array off the 16-byte grid."""
    B, D, lens = 4, 64, [0, 40]
    rng = np.random.default_rng(n)
    P, cnt = [0, 70, 0, 5], [n, n - 1, n, 0]
    S = 70 + n
    shared, K0, V0 = _filled(A, rng, 2, H, 44, D)
    cache, K, V = _filled(A, rng, B, H, S, D)
    mask = rng.random((B, n, n)) < 0.3
    mask[0, 2] = False                                          # without a prefix: sees nothing
    mask[2] = False                                             # sees the prefix alone
    depth = rng.integers(0, 9, (B, n))
    wide = torch.zeros(B, n, Hq * D + 3, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    q = wide[:, :, 1:1 + Hq * D].unflatten(-1, (Hq, D))
    q.copy_(_torch(rng.standard_normal((B, n, Hq, D)), dtype))
    if passes == 2:
        shared = _roomy(A, shared)
    for window, sinks in ((0, 0), (6, 2), (60, 0), (2_000_000, 0)):
        r = A.kv4_shared_attention(q, shared, _i32(lens), cache, 0, _i32(P), mask=_words(mask), depth=_i32(depth), count=_i32(cnt), scale=0.21,
                                   window=window, sinks=sinks)
        _check(r, _f64(q), (K0, V0), lens, (K, V), P, cnt, dtype, 0.21, mask, depth, window, sinks)
        assert not r["out"][0, 2].any() and torch.isneginf(r["lse"][0, 2]).all() and not r["out"][3].any()


@pytest.mark.parametrize("passes", [1, 2])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40])
def test_sequences_outside_the_caches(A, dtype, n, passes):
    B, Hq, H, D, S, S0 = 8, 4, 2, 128, 60, 30
    rng = np.random.default_rng(3)
    shared, K0, V0 = _filled(A, rng, 4, H, S0, D)
    cache, K, V = _filled(A, rng, B, H, S, D)
    q = _torch(rng.standard_normal((B, n, Hq, D)), dtype)
    if passes == 2:
        shared = _roomy(A, shared)
    lens, P, cnt = [30, -1, shared.shape[3] + 1, 4], [-1, 20, 3, 4, 5, 6, 61 - n, 0], [n, n, n, n, n, n, n, n + 1]
    r = A.kv4_shared_attention(q, shared, _i32(lens), cache, 0, _i32(P), count=_i32(cnt))
    np.testing.assert_array_equal(r["status"].cpu().numpy(), [8, 0, 8, 8, 8, 8, 8, 8])
    for b in (0, 2, 3, 4, 5, 6, 7):
        assert not r["out"][b].any() and torch.isneginf(r["lse"][b]).all()
    _check({key: r[key][1:2] for key in ("out", "lse")}, _f64(q)[1:2], (K0, V0), [30], (K[1:2], V[1:2]), [20], [n], dtype, D ** -0.5)


@pytest.mark.parametrize("passes", [1, 2])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_bad_query_spoils_its_own_row(A, n, dtype, passes):
    B, Hq, H, D, S = 24, 4, 2, 64, 100
    rng = np.random.default_rng(4)
    shared, _, _ = _filled(A, rng, 1, H, 90, D)
    cache, _, _ = _filled(A, rng, B, H, S, D)
    if passes == 2:
        shared = _roomy(A, shared)
    q = _torch(rng.standard_normal((B, n, Hq, D)), dtype)
    P, cnt = _i32(list(range(B))), _i32([n] * (B - 1) + [n - 1])
    call = lambda x: A.kv4_shared_attention(x, shared, _i32([80]), cache, 0, P, count=cnt)  # noqa: E731
    clean = call(q)
    for bad in (float("nan"), float("inf")):
        p = q.clone()
        p[1, n // 2, 3, 5] = bad
        p[B - 1, n - 1] = bad                                   # padding: nobody's
        r = call(p)
        assert torch.isnan(r["out"][1, n // 2, 3]).all()
        for key in ("out", "lse"):
            a, b = r[key].clone(), clean[key].clone()
            a[1, n // 2, 3] = b[1, n // 2, 3] = 0
            assert torch.equal(a, b)


@pytest.mark.parametrize("passes", [1, 2])
@pytest.mark.parametrize("n,B", [(1, 3), (1, 50), (40, 3)])
def test_it_is_the_attention_over_one_cache(A, n, B, passes):
    """Against kv4_attention over caches that hold the prefix's rows before their own, moved as bytes."""
    Hq, H, D, S0, lens = 8, 2, 128, 500, [437]
    rng = np.random.default_rng(B)
    shared, _, _ = _filled(A, rng, 1, H, S0, D)
    cache, _, _ = _filled(A, rng, B, H, 200 + n, D)
    P = rng.integers(0, 200, B)
    whole = A.kv4_cache(1, B, H, S0 + 200 + n, D)
    whole[:, :, :, :437] = shared[:, :, :, :437]
    whole[:, :, :, 437:437 + 200 + n] = cache
    q = _torch(rng.standard_normal((B, n, Hq, D)), "bf16")
    if passes == 2:
        shared = _roomy(A, shared)
    for window, sinks in ((0, 0), (300, 4)):
        r = A.kv4_shared_attention(q, shared, _i32(lens), cache, 0, _i32(P), window=window, sinks=sinks)
        one = A.kv4_attention(q, whole, 0, _i32(437 + P), window=window, sinks=sinks)
        # two computations, each within the bound of the other tests: weights and results of 2^-8 each
        assert (r["out"].float() - one["out"].float()).abs().max() <= 4 * 2.0 ** -8 * 4
        assert (r["lse"] - one["lse"]).abs().max() <= 2.0 ** -17 * 40


@pytest.mark.parametrize("passes", [1, 2])
def test_graphs_streams_and_workspaces(A, passes):
    B, n, Hq, H, D = 12, 1, 8, 2, 128
    rng = np.random.default_rng(9)
    shared, _, _ = _filled(A, rng, 2, H, 3000, D)
    cache, _, _ = _filled(A, rng, B, H, 300, D)
    q = _torch(rng.standard_normal((B, n, Hq, D)), "bf16")
    lens, P = _i32([3000, 2500]), _i32(list(range(0, 12 * 20, 20)))
    if passes == 2:
        shared = _roomy(A, shared)
    want = A.kv4_shared_attention(q, shared, lens, cache, 0, P)
    need = A.kv4_shared_workspace_bytes(B, 2, n, Hq, H, D)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    r = A.kv4_shared_attention(q, shared, lens, cache, 0, P, workspace=ws[:need])
    torch.cuda.synchronize()
    assert torch.equal(r["out"], want["out"]) and torch.equal(r["lse"], want["lse"]) and (ws[need:] == 255).all()
    with pytest.raises(A.AcespecError):
        A.kv4_shared_attention(q, shared, lens, cache, 0, P, workspace=ws[:need - 16])
    base = torch.cuda.memory_allocated()
    for s in [torch.cuda.Stream() for _ in range(3)]:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            r = A.kv4_shared_attention(q, shared, lens, cache, 0, P)
        s.synchronize()
        assert torch.equal(r["out"], want["out"])
        del r
    assert torch.cuda.memory_allocated() <= base
    # two graphs, replayed in turns and at once, each with its own results
    graphs, outs = [], []
    for scale in (0.1, 0.3):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(A.kv4_shared_attention(q, shared, lens, cache, 0, P, scale=scale))
        graphs.append(g)
    wants = [A.kv4_shared_attention(q, shared, lens, cache, 0, P, scale=s) for s in (0.1, 0.3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, wants):
        assert torch.equal(o["out"], w["out"]) and torch.equal(o["lse"], w["lse"])
    lens.copy_(_i32([100, 7]))                                 # the captured call reads the lengths when it runs
    graphs[0].replay()
    fresh = A.kv4_shared_attention(q, shared, lens, cache, 0, P, scale=0.1)
    torch.cuda.synchronize()
    assert torch.equal(outs[0]["out"], fresh["out"])


def test_the_binding_refuses(A):
    q, shared, cache = torch.zeros(4, 1, 2, 64, device="cuda"), A.kv4_cache(1, 2, 1, 8, 64), A.kv4_cache(1, 4, 1, 8, 64)
    lens, P = _i32([1, 1]), _i32([0] * 4)
    A.kv4_shared_attention(q, shared, lens, cache, 0, P)
    for kw in (dict(shared=A.kv4_cache(1, 3, 1, 8, 64)), dict(shared=A.kv4_cache(1, 2, 2, 8, 64)), dict(shared=A.kv4_cache(1, 2, 1, 8, 128)),
               dict(shared=shared[:, :, :, ::2]), dict(shared=shared.cpu()), dict(shared=None), dict(shared_len=P), dict(shared_len=lens.long()),
               dict(shared_len=None), dict(prefix_len=lens)):
        with pytest.raises(ValueError):
            A.kv4_shared_attention(**{**dict(q=q, shared=shared, shared_len=lens, cache=cache, layer=0, prefix_len=P), **kw})
    with pytest.raises(A.AcespecError):
        A.kv4_shared_attention(q, shared, lens, cache, 1, P)


def test_another_device_is_refused(A, monkeypatch):
    q, cache = torch.zeros(1, 1, 1, 64, device="cuda"), A.kv4_cache(1, 1, 1, 8, 64)
    monkeypatch.setattr(A, "_current_device", lambda: 1)     # as if another GPU were the current one
    with pytest.raises(ValueError, match="current device"):
        A.kv4_shared_attention(q, cache, _i32([1]), cache, 0, _i32([0]))
