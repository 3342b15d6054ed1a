"""The 4-bit KV cache and its attention against float64 numpy (oracle/kv4.py).

Bounds, from the arithmetic and not from runs.  The cache's values are exact,
so the bytes written and the numbers read are compared bit for bit.  In the
attention every product with a cache value is exact and what rounds is:
  - a score's sum of D products in float32: at most 2^-20 of M, the largest
    scale * sum |q| |k| (some 2^-23 for each of the sum's partial sums);
    twice that, relative, in a weight and in the sum of the weights;
  - the weights' exponentials and sums, and their products' sums: 2^-17;
  - bfloat16 queries: the weights' rounding, 2^-8, and the result's, 2^-8 (half
    a unit of eight significant bits is up to 2^-8 of the number).
All are relative to A = sum of the weights times |v| of the output's channel.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import kv4 as O  # noqa: E402


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_02514_gb300 as A
    A.load()
    return A


def _torch(x, dtype):
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()
    return t if dtype == "f32" else t.to(torch.bfloat16)


def _f64(t):
    return t.double().cpu().numpy()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _numbers(rng, shape):
    """Rows of which some groups are large, tiny, zero or tied."""
    x = rng.standard_normal(shape) * np.exp(1.5 * rng.standard_normal(shape[:-1] + (1,)))
    g = x.reshape(shape[:-1] + (8, shape[-1] // 8))
    kind = rng.integers(0, 12, g.shape[:-1])
    g[kind == 0] = 0.0
    g[kind == 1] *= 1e-30
    g[kind == 2] *= 3e5
    g[kind == 3] = np.sign(g[kind == 3])                       # ties of both signs
    g[kind == 4] = np.round(g[kind == 4] * 4) / 4              # quotients on halves
    return x


# -- writing and reading ------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,n,H,S,lay", [(1, 1, 1, 1, "dense"), (3, 17, 2, 40, "dense"), (2, 9, 3, 30, "fused"), (2, 6, 1, 30, "odd"),
                                         (7, 700, 1, 720, "fused")])
def test_rows_are_the_definitions(A, dtype, D, B, n, H, S, lay):
    rng = np.random.default_rng(D + B + n)
    k, v = _numbers(rng, (B, n, H, D)), _numbers(rng, (B, n, H, D))
    tk, tv = _torch(k, dtype), _torch(v, dtype)
    k64, v64 = _f64(tk), _f64(tv)
    if lay != "dense":       # a slice of a wider array; "odd": off the 16-byte grid
        extra = 1 if lay == "odd" else 0
        wide = torch.zeros(B, n, 3 * H * D + extra + 8, dtype=tk.dtype, device="cuda")
        wk = wide[:, :, H * D + extra:2 * H * D + extra].unflatten(-1, (H, D))
        wv = wide[:, :, 2 * H * D + extra:3 * H * D + extra].unflatten(-1, (H, D))
        wk.copy_(tk)
        wv.copy_(tv)
        tk, tv = wk, wv
    cache = A.kv4_cache(2, B, H, S, D)
    cache.fill_(0xAB)
    start = rng.integers(0, S - n + 1, B)
    status = A.kv4_append(cache, 1, tk, tv, _i32(start))
    got = cache.cpu().numpy()
    want = np.full_like(got, 0xAB)
    some = range(B) if B * n * H < 200 else [0, B - 1]
    for b in some:
        for p, x in ((2, k64), (3, v64)):
            want[p, b, :, start[b]:start[b] + n] = O.rows_of(x[b].swapaxes(0, 1))
        np.testing.assert_array_equal(got[:, b], want[:, b])
    assert not status.any()
    for dt, name in ((torch.float32, "f32"), (torch.bfloat16, "bf16")):
        back = A.kv4_read(cache, 1, _i32(start), n, dtype=dt)
        for b in some:
            for key, p in (("k", 2), ("v", 3)):
                vals = O.values_of(want[p, b, :, start[b]:start[b] + n]).swapaxes(0, 1)
                np.testing.assert_array_equal(_f64(back[key][b]), vals)
    # half a step, or 1.25 for what lies beyond 7.5 steps on the other arm (|a| is up to 8.25 steps, the arm ends at 7)
    if dtype == "f32":
        x = k64[0]
        step = np.abs([[[O.step_of(x[i, h, g * (D // 8):(g + 1) * (D // 8)]) for g in range(8)] for h in range(H)] for i in range(n)])
        off = np.abs(_f64(A.kv4_read(cache, 1, _i32(start), n, dtype=torch.float32)["k"][0]) - x).reshape(n, H, 8, -1)
        big = np.abs(x).reshape(n, H, 8, -1).max(-1)
        assert (off <= 1.25 * np.maximum(step, 2.0 ** -90)[..., None] + np.maximum(big - O.CAP, 0)[..., None]).all()


def test_any_bytes_are_finite_numbers(A):
    rng = np.random.default_rng(5)
    for D in (64, 128):
        cache = torch.from_numpy(rng.integers(0, 256, (2, 2, 2, 33, D // 2 + 16), dtype=np.uint8)).cuda()
        cache[:, :, :, :4] = 255
        back = A.kv4_read(cache, 0, _i32([0, 0]), 33, dtype=torch.float32)
        for p, key in ((0, "k"), (1, "v")):
            got = _f64(back[key])
            assert np.isfinite(got).all()
            want = O.values_of(cache[p].cpu().numpy()).transpose(0, 2, 1, 3)
            normal = (np.abs(want) >= 2.0 ** -100) | (want == 0)      # what no row is written with may read as 0
            np.testing.assert_array_equal(got[normal], want[normal])


def test_bad_numbers_and_places(A):
    B, n, H, D, S = 3, 5, 2, 64, 12
    x = torch.randn(B, n, H, D, device="cuda")
    x[0, 1, 1, 3] = float("nan")
    x[0, 3, 0, 9] = float("inf")
    y = torch.randn(B, n, H, D, device="cuda")
    y[1, 4, 1, 60] = -float("inf")
    cache = A.kv4_cache(1, B, H, S, D)
    start, count = _i32([2, 9, -2]), _i32([4, 5, 5])
    st = A.kv4_append(cache, 0, x, y, start, count=count).cpu().numpy()
    R, N = A.ROW_RANGE, A.ROW_NONFINITE
    np.testing.assert_array_equal(st, [[0, N, 0, N, 0], [0, 0, 0, R, R], [R, R, 0, 0, 0]])
    rows = cache.cpu().numpy()
    assert not rows[:, 0, :, 6:].any() and not rows[:, 0, :, :2].any()        # the padding token too
    clean = np.nan_to_num(x.double().cpu().numpy(), nan=0.0, posinf=O.CAP, neginf=-O.CAP)
    np.testing.assert_array_equal(rows[0, 0, :, 2:6], O.rows_of(clean[0, :4].swapaxes(0, 1)))
    back = A.kv4_read(cache, 0, start, n, dtype=torch.float32)["k"]
    assert not back[1, 3:].any() and not back[2, :2].any() and back[1, :3].any(-1).all()


# -- attention ----------------------------------------------------------------
def _tree_bits(F, L):
    K = len(F)
    n = K + sum(F) * L
    m, depth = np.zeros((n, n), bool), list(range(K))
    for q in range(K):
        m[q, :q + 1] = True
    at = K
    for d, f in enumerate(F):
        for _ in range(f):
            for o in range(L):
                m[at + o, :d] = True
                m[at + o, at:at + o + 1] = True
                depth.append(d + o)
            at += L
    return m, np.array(depth)


def _words(m):
    n = m.shape[-1]
    bits = np.zeros(m.shape[:-1] + ((n + 31) // 32 * 32,), bool)
    bits[..., :n] = m
    w = (bits.reshape(*m.shape[:-1], -1, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    return torch.from_numpy(w.view(np.int32)).cuda()


def _filled(A, rng, B, H, S, D, layers=1, layer=0):
    """A cache of S written positions and its numbers K, V [B, H, S, D]."""
    k, v = rng.standard_normal((B, S, H, D)), rng.standard_normal((B, S, H, D))
    k *= np.exp(0.5 * rng.standard_normal((1, 1, H, D)))
    cache = A.kv4_cache(layers, B, H, S, D)
    zero = _i32([0] * B)
    A.kv4_append(cache, layer, _torch(k, "f32"), _torch(v, "f32"), zero)
    back = A.kv4_read(cache, layer, zero, S, dtype=torch.float32)
    return cache, _f64(back["k"]).swapaxes(1, 2), _f64(back["v"]).swapaxes(1, 2)


def _compare(r, q, K, V, P, cnt, dtype, scale, mask=None, depth=None, window=0, sinks=0, rows=None, S=None):
    B, n, Hq, D = q.shape
    H = K.shape[1]
    out, lse = _f64(r["out"]), _f64(r["lse"])
    for b in range(B):
        top = min(S or K.shape[2], max(P[b] + cnt[b], 1))
        m = mask[b] if mask is not None and mask.ndim == 3 else mask
        d = depth[b] if depth is not None and depth.ndim == 2 else depth
        ok = O.visible(P[b], cnt[b], n, top, m, d, window, sinks)
        for hq in range(Hq):
            h = hq // (Hq // H)
            w, z, mag, M = O.attend(q[b, :, hq], K[b, h, :top], V[b, h, :top], ok, scale)
            rel = 4 * 2.0 ** -20 * (M + 1) + 2.0 ** -17 + (2.0 ** -7 if dtype == "bf16" else 0.0)
            off = np.abs(out[b, :, hq] - w)
            assert (off <= rel[:, None] * mag + 1e-30).all(), (b, hq, float((off / (rel[:, None] * mag + 1e-30)).max()))
            seen = np.isfinite(z)
            np.testing.assert_array_equal(np.isneginf(lse[b, :, hq]), ~seen)
            assert (np.abs(lse[b, seen, hq] - z[seen]) <= 2.0 ** -19 * (M[seen] + np.abs(z[seen]) + 1)).all()


# B, n, Hq, H, D, cached positions, form, window, sinks
SHAPES = [
    (2, 1, 1, 1, 64, [0, 37], "causal", 0, 0),                 # one head, an empty cache
    (3, 1, 8, 8, 128, [1, 31, 32], "causal", 0, 0),            # every head its own keys
    (2, 1, 12, 4, 64, [300, 1023], "causal", 0, 0),            # three heads share keys
    (1, 1, 40, 8, 128, [2500], "causal", 0, 0),
    (2, 1, 16, 1, 128, [700, 90], "causal", 0, 0),             # one key head
    (1, 1, 71, 1, 64, [260], "causal", 0, 0),                  # more rows than a tensor tile's half
    (2, 5, 4, 2, 64, [100, 3], "causal", 0, 0),
    (2, 3, 8, 1, 128, [513, 0], "causal", 0, 0),
    (1, 33, 4, 4, 128, [95], "causal", 0, 0),
    (2, 64, 2, 1, 64, [127, 64], "causal", 0, 0),              # 128 rows
    (1, 129, 2, 2, 128, [1], "causal", 0, 0),                  # one row above a tile
    (2, 100, 6, 2, 64, [200, 411], "causal", 0, 0),            # 300 rows
    (1, 520, 2, 2, 128, [130], "causal", 0, 0),
    (2, 1, 8, 2, 128, [900, 40], "causal", 100, 4),            # windows
    (2, 1, 4, 4, 64, [333, 5], "causal", 1, 0),
    (1, 40, 4, 2, 64, [500], "causal", 64, 3),
    (1, 200, 2, 1, 128, [300], "causal", 33, 1),
    (2, 300, 2, 2, 64, [0, 129], "causal", 128, 5),
    (2, 0, 4, 2, 128, [50, 0], "tree", 0, 0),
    (1, 0, 8, 2, 64, [777], "tree", 0, 0),
    (2, 0, 16, 2, 128, [300, 129], "bigtree", 0, 0),
    (2, 0, 4, 2, 64, [100, 9], "tree", 4, 2),
    (1, 0, 16, 2, 128, [260], "bigtree", 7, 130),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_attention_is_the_definition(A, case, dtype):
    B, n, Hq, H, D, P, form, window, sinks = case
    rng = np.random.default_rng(B + 7 * n + Hq + P[0])
    mask = depth = None
    if form != "causal":
        mask, depth = _tree_bits([2, 1, 2], 2) if form == "tree" else _tree_bits([4] * 8, 1)
        n = len(depth)
        words, dev_depth = _words(mask), _i32(depth)
        if form == "bigtree" and not window:
            aw, ad = A.tree_mask([4] * 8, 1)                    # the library's own mask
            assert torch.equal(aw, words) and torch.equal(ad, dev_depth)
    cnt = [n, max(0, n - 3)][:B] + [n] * (B - 2)
    S = max(P) + n + 3
    cache, K, V = _filled(A, rng, B, H, S, D, layers=2, layer=1)
    for b in range(B):
        cache[:, b, :, P[b] + cnt[b]:] = 255                    # bytes nobody wrote
    q = _torch(rng.standard_normal((B, n, Hq, D)) * 0.8, dtype)
    r = A.kv4_attention(q, cache, 1, _i32(P), mask=None if mask is None else words, depth=None if mask is None else dev_depth,
                        count=_i32(cnt), window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert not r["status"].any()
    _compare(r, _f64(q), K, V, P, cnt, dtype, D ** -0.5, mask, depth, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,H", [(6, 4, 2), (50, 6, 2)])
def test_any_mask_any_strides(A, dtype, n, Hq, H):
    """A mask and depths of every sequence, rows that see nothing, another
    scale, and queries inside a wider array off the 16-byte grid."""
    B, D = 3, 64
    rng = np.random.default_rng(n)
    P, cnt = [0, 70, 0], [n, n - 1, n]
    S = 70 + n
    cache, K, V = _filled(A, rng, B, H, S, D)
    mask = rng.random((B, n, n)) < 0.3
    mask[0, 2] = False                                          # with an empty prefix: sees nothing
    mask[2] = False
    depth = rng.integers(0, 9, (B, n))
    wide = torch.zeros(B, n, Hq * D + 3, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    q = wide[:, :, 1:1 + Hq * D].unflatten(-1, (Hq, D))
    q.copy_(_torch(rng.standard_normal((B, n, Hq, D)), dtype))
    for window, sinks in ((0, 0), (6, 2)):
        r = A.kv4_attention(q, cache, 0, _i32(P), mask=_words(mask), depth=_i32(depth), count=_i32(cnt), scale=0.21, window=window,
                            sinks=sinks)
        _compare(r, _f64(q), K, V, P, cnt, dtype, 0.21, mask, depth, window, sinks)
        assert not r["out"][2].any() and torch.isneginf(r["lse"][2]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sequences_outside_the_cache(A, dtype):
    B, n, Hq, H, D, S = 4, 2, 4, 2, 128, 50
    rng = np.random.default_rng(3)
    cache, K, V = _filled(A, rng, B, H, S, D)
    q = _torch(rng.standard_normal((B, n, Hq, D)), dtype)
    r = A.kv4_attention(q, cache, 0, _i32([-1, 49, 20, 20]), count=_i32([2, 2, 3, 2]))
    np.testing.assert_array_equal(r["status"].cpu().numpy(), [8, 8, 8, 0])
    assert not r["out"][:3].any() and torch.isneginf(r["lse"][:3]).all()
    _compare({key: r[key][3:] for key in ("out", "lse")}, _f64(q)[3:], K[3:], V[3:], [20], [2], dtype, D ** -0.5)


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_bad_query_spoils_its_own_row(A, n, dtype):
    B, Hq, H, D, S = 2, 4, 2, 64, 200
    rng = np.random.default_rng(4)
    cache, K, V = _filled(A, rng, B, H, S, D)
    q = _torch(rng.standard_normal((B, n, Hq, D)), dtype)
    clean = A.kv4_attention(q, cache, 0, _i32([100, 60]))
    for bad in (float("nan"), float("inf")):
        p = q.clone()
        p[1, n // 2, 3, 5] = bad
        r = A.kv4_attention(p, cache, 0, _i32([100, 60]))
        assert torch.isnan(r["out"][1, n // 2, 3]).all()
        for key in ("out", "lse"):
            a, b = r[key].clone(), clean[key].clone()
            a[1, n // 2, 3] = b[1, n // 2, 3] = 0
            assert torch.equal(a, b), key


@pytest.mark.parametrize("dtype,B,n,Hq,H,D,P", [("bf16", 1, 1, 8, 2, 128, 20000), ("f32", 2, 1, 2, 2, 64, 9000), ("bf16", 1, 24, 8, 1, 128, 9000),
                                                ("bf16", 2, 2, 64, 1, 64, 3333)])
def test_long_caches(A, dtype, B, n, Hq, H, D, P):
    """Keys enough that a row's work is split and joined; large scores far apart."""
    rng = np.random.default_rng(P)
    cache, K, V = _filled(A, rng, B, H, P + n, D)
    q = _torch(rng.standard_normal((B, n, Hq, D)) * 3.0, dtype)
    Ps = [P - 777 * b for b in range(B)]
    r = A.kv4_attention(q, cache, 0, _i32(Ps))
    _compare(r, _f64(q), K, V, Ps, [n] * B, dtype, D ** -0.5)
    again = A.kv4_attention(q, cache, 0, _i32(Ps))
    for key in ("out", "lse"):
        assert torch.equal(r[key], again[key])                  # no order of arrival in the result


@pytest.mark.parametrize("D", [64, 128])
def test_rows_move_with_compact_kv(A, D):
    """The tree's rows are moved as they are, and the attention after the move
    is that over a cache written in the new order."""
    B, H, S, F, L = 3, 2, 60, [2, 1, 2], 2
    K, n = len(F), len(F) + sum(F) * L
    rng = np.random.default_rng(D)
    cache, _, _ = _filled(A, rng, B, H, S, D, layers=2)
    k = _torch(rng.standard_normal((B, n, H, D)), "bf16")
    v = _torch(rng.standard_normal((B, n, H, D)), "bf16")
    t = _i32([20, 7, 33])
    for layer in (0, 1):
        A.kv4_append(cache, layer, k, v, t)
    before = cache.clone()
    pi, slot = _i32([1, 0, K]), _i32([2, 1, -2])
    new_len = A.compact_kv(cache, t, pi, slot, K, L)
    np.testing.assert_array_equal(new_len.cpu().numpy(), [20 + 1 + L, 7 + 0 + L, 33 + K])
    for b, (t0, p, s) in enumerate([(20, 1, 2), (7, 0, 1)]):
        assert torch.equal(cache[:, b, :, t0 + p:t0 + p + L], before[:, b, :, t0 + K + s * L:t0 + K + (s + 1) * L])
    q = _torch(rng.standard_normal((B, 1, 4, D)), "bf16")
    one = _torch(rng.standard_normal((B, 1, H, D)), "bf16")
    A.kv4_append(cache, 0, one, one, new_len)
    r = A.kv4_attention(q, cache, 0, new_len)
    back = A.kv4_read(cache, 0, _i32([0] * B), S, dtype=torch.float32)
    _compare(r, _f64(q), _f64(back["k"]).swapaxes(1, 2), _f64(back["v"]).swapaxes(1, 2), new_len.tolist(), [1] * B, "bf16", D ** -0.5)


def test_another_stream_and_a_graph(A):
    B, n, Hq, H, D, S = 2, 7, 8, 2, 128, 400
    rng = np.random.default_rng(8)
    cache, _, _ = _filled(A, rng, B, H, S, D)
    q = _torch(rng.standard_normal((B, n, Hq, D)), "bf16")
    k = _torch(rng.standard_normal((B, n, H, D)), "bf16")
    P = _i32([300, 11])
    torch.cuda.synchronize()
    ref_cache = cache.clone()
    A.kv4_append(ref_cache, 0, k, k, P)
    ref = A.kv4_attention(q, ref_cache, 0, P)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        A.kv4_append(cache, 0, k, k, P)
        r = A.kv4_attention(q, cache, 0, P)
    s.synchronize()
    assert torch.equal(cache, ref_cache) and torch.equal(r["out"], ref["out"])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        A.kv4_append(cache, 0, k, k, P)
        r = A.kv4_attention(q, cache, 0, P)
    cache.zero_()
    cache.copy_(ref_cache)
    r["out"].zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(r["out"], ref["out"])


def test_offsets_beyond_32_bits(A):
    """The last sequence's rows of a plane and the second layer lie past 2^32 bytes."""
    B, H, D, S = 65, 1, 128, 830000
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    cache = torch.empty(4, B, H, S, D // 2 + 16, dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(9)
    n, far = 40, S - 41
    k, v = rng.standard_normal((B, n, H, D)), rng.standard_normal((B, n, H, D))
    start = [0] * (B - 1) + [far]
    A.kv4_append(cache, 1, _torch(k, "f32"), _torch(v, "f32"), _i32(start))
    np.testing.assert_array_equal(cache[3, B - 1, 0, far:far + n].cpu().numpy(), O.rows_of(_f64(_torch(v, "f32"))[B - 1, :, 0]))
    back = A.kv4_read(cache, 1, _i32(start), n, dtype=torch.float32)
    kb, vb = _f64(back["k"]), _f64(back["v"])
    q = _torch(rng.standard_normal((B, n, 2, D)), "bf16")
    pre = [0] * (B - 1) + [far]
    for new in (1, n):
        r = A.kv4_attention(q[:, :new].contiguous(), cache, 1, _i32(pre), window=new, sinks=0)
        for hq in range(2):
            ok = np.tril(np.ones((new, new), bool))
            w, z, mag, M = O.attend(_f64(q)[B - 1, :new, hq], kb[B - 1, :new, 0], vb[B - 1, :new, 0], ok, D ** -0.5)
            if new == 1:
                assert (np.abs(_f64(r["out"])[B - 1, :, hq] - w) <= 2.0 ** -7 * mag).all()
    A.kv4_append(cache, 1, _torch(k, "f32"), _torch(v, "f32"), _i32([0] * (B - 1) + [far]))
    r = A.kv4_attention(q, cache, 1, _i32(pre), window=1)
    np.testing.assert_array_equal(_f64(r["out"])[B - 1], _f64(back["v"].to(torch.bfloat16))[B - 1].repeat(2, 1))
