"""rotate_qk and kv4_append_rotated against float64 numpy (oracle/turn.py).

Bounds, from the arithmetic and not from runs.  In units u = 2^-24 a number is
off by at most 16 u of the length h of its pair (after the norm): the sum of
squares 9 u, half of which shows in the root, its mean with eps 0.5 u, the root,
its product with the weight and with the number 1 u each; two products and
their sum 2 u; the sine and cosine 3.7 u of h; the scale's two roundings.
Channels that do not turn are within that of themselves.  bfloat16 results are
rounded once more, by at most 2^-8 of the number.  The cache's numbers are
compared bit for bit: the codes are those of the 64-bit numbers.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import turn as O  # noqa: E402


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


DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _i32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


def _f64(t):
    return t.double().cpu().numpy()


def _heads(rng, B, n, counts, D, dtype, lay):
    """Queries, keys and values as one projection gives them: strided views of one array; "odd": off the 16-byte grid."""
    heads = sum(counts)
    extra = {"fused": 0, "odd": 1, "dense": 0}[lay]
    x = rng.standard_normal((B, n, heads * D + extra)) * np.exp(rng.standard_normal((B, n, 1)))
    wide = torch.from_numpy(x.astype(np.float32)).cuda().to(DT[dtype])[:, :, extra:].unflatten(-1, (heads, D))
    parts = wide.split(list(counts), dim=2)
    return [p.contiguous() for p in parts] if lay == "dense" else list(parts)


def _freq(R, theta=10000.0):
    return torch.from_numpy((theta ** (-np.arange(R // 2) / (R // 2))).astype(np.float32)).cuda()


def _close(got, z, h, dtype):
    off = np.abs(_f64(got) - z)
    bound = 16 * 2.0 ** -24 * h * (1 + 2.0 ** -8) + (2.0 ** -8 * np.abs(z) if dtype == "bf16" else 0.0)
    assert (off <= bound).all(), (off / np.maximum(bound, 1e-300)).max()


def _weights(rng, kind, heads, D, dtype):
    if kind == "none":
        return None
    shape = (D,) if kind in ("one", "one f32") else (heads, D)
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(shape)).astype(np.float32)).cuda()
    return w if kind == "one f32" else w.to(DT[dtype])


CASES = [  # B, n, Hq, H, R / (D / 4), axes, interleaved, weights, layout
    (1, 1, 1, 1, 4, 1, False, "one", "dense"), (1, 1, 32, 8, 4, 1, False, "one", "fused"), (3, 17, 5, 1, 2, 1, True, "each", "odd"),
    (2, 7, 12, 4, 1, 3, False, "none", "fused"), (2, 33, 3, 3, 3, 4, True, "one f32", "fused"), (1, 700, 8, 2, 4, 3, False, "each", "fused"),
    (5, 541, 6, 2, 2, 2, False, "one", "odd"), (1, 5000, 2, 1, 4, 3, True, "off", "dense"), (2, 3000, 3, 1, 3, 1, False, "off", "fused")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,n,Hq,H,quarters,axes,inter,weights,lay", CASES)
def test_rotation_is_the_definition(A, dtype, D, B, n, Hq, H, quarters, axes, inter, weights, lay):
    rng = np.random.default_rng(D + n + Hq)
    R = quarters * D // 4
    q, k = _heads(rng, B, n, (Hq, H), D, dtype, lay)
    f = _freq(R)
    eps = None if weights == "off" else 1e-5
    qw, kw = (None, None) if weights == "off" else (_weights(rng, weights, Hq, D, dtype), _weights(rng, weights, H, D, dtype))
    start = rng.integers(-50, 200000, B)
    turn = dict(q_weight=qw, k_weight=kw, eps=eps, interleaved=inter, scale=1.0 if n % 2 else 1.2079)
    if axes == 1:
        pos, ax = (start[:, None] + np.arange(n))[None], None
        r = A.rotate_qk(q, k, f, start=_i32(start), **turn)
    else:
        pos = rng.integers(-1000, 1 << 20, (axes, B, n))
        ax = rng.integers(-1, axes + 1, R // 2)              # those outside take the nearest
        r = A.rotate_qk(q, k, f, positions=_i32(pos), axes=_i32(ax), **turn)
    for x, w, key in ((q, qw, "q"), (k, kw, "k")):
        z, h = O.turned(_f64(x), _f64(f), pos, ax, None if w is None else _f64(w), eps, inter, turn["scale"])
        _close(r[key], z, h, dtype)


def test_far_positions_keep_their_angles(A):
    """Positions up to the type's ends, where float32 would have no angle left."""
    rng = np.random.default_rng(1)
    pos = np.array([[2 ** 20 + 1, 2 ** 24 + 3, 2 ** 31 - 1, -2 ** 31, 0, -7]])
    q, k = _heads(rng, 1, 6, (2, 1), 128, "f32", "dense")
    f = _freq(128)
    r = A.rotate_qk(q, k, f, positions=_i32(pos))
    z, h = O.turned(_f64(q), _f64(f), pos[None])
    _close(r["q"], z, h, "f32")
    assert torch.equal(r["q"][0, 4], q[0, 4]) and torch.equal(r["k"][0, 4], k[0, 4])     # position 0 turns nothing


@pytest.mark.parametrize("D", [64, 128])
def test_trees_and_sequences_of_depths(A, D):
    rng = np.random.default_rng(2)
    _, depth = A.tree_mask([2, 1, 0], 2)
    n = len(depth)
    q, k = _heads(rng, 3, n, (4, 2), D, "bf16", "fused")
    f, start = _freq(D), np.array([0, 77, 100000])
    each = torch.stack([depth, depth * 2, depth + 5])
    for dep in (depth, each):
        r = A.rotate_qk(q, k, f, start=_i32(start), depth=dep)
        d = np.broadcast_to(dep.cpu().numpy(), (3, n))
        z, h = O.turned(_f64(k), _f64(f), (start[:, None] + d)[None])
        _close(r["k"], z, h, "bf16")


def test_in_place_and_strided_outputs(A):
    rng = np.random.default_rng(3)
    q, k = _heads(rng, 2, 9, (6, 2), 64, "bf16", "fused")
    before = q[0, 0, 0].clone()
    f, start = _freq(32), _i32([3, 90])
    want = A.rotate_qk(q, k, f, start=start, eps=1e-6)
    wide = torch.full((9, 2, 3, 6, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    out = wide[:, :, 1].transpose(0, 1)                        # other strides, and numbers in between that stay
    r = A.rotate_qk(q, k, f, start=start, eps=1e-6, out=dict(q=out))
    assert r["q"] is out and torch.equal(out, want["q"]) and torch.equal(r["k"], want["k"])
    assert (wide[:, :, 0] == 7).all() and (wide[:, :, 2] == 7).all() and torch.equal(before, q[0, 0, 0])
    r = A.rotate_qk(q, k, f, start=start, eps=1e-6, out=dict(q=q, k=k))
    assert r["q"] is q and torch.equal(q, want["q"]) and torch.equal(k, want["k"])
    with pytest.raises(ValueError, match="layout"):
        A.rotate_qk(want["q"], want["k"], f, start=start, out=dict(q=want["q"].view(9, 2, 6, 64).transpose(0, 1)))
    with pytest.raises(A.AcespecError):
        A.rotate_qk(want["q"], want["k"], f, start=start, out=dict(q=torch.empty(1, 9, 6, 64, device="cuda", dtype=torch.bfloat16).expand(2, 9, 6, 64)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_of_many_tokens(A, dtype):
    """Rows are read ahead of those that are written, of several tokens a warp."""
    rng = np.random.default_rng(13)
    q, k = _heads(rng, 2, 9000, (5, 3), 64, dtype, "fused")
    f, start = _freq(64), _i32([1, 70000])
    want = A.rotate_qk(q, k, f, start=start, eps=1e-6)
    A.rotate_qk(q, k, f, start=start, eps=1e-6, out=dict(q=q, k=k))
    assert torch.equal(q, want["q"]) and torch.equal(k, want["k"])
    for b, i in ((0, 0), (1, 8999), (1, 3), (0, 6000)):
        one = A.rotate_qk(want["q"][b:b + 1, i:i + 1], want["k"][b:b + 1, i:i + 1], f, start=start[b:b + 1] + i)
        many = A.rotate_qk(want["q"], want["k"], f, start=start)
        assert torch.equal(one["q"][0, 0], many["q"][b, i]) and torch.equal(one["k"][0, 0], many["k"][b, i])


def test_rows_do_not_hang_on_their_neighbours(A):
    """A token's numbers are the same bits alone and in a batch of any size."""
    rng = np.random.default_rng(4)
    q, k, v = _heads(rng, 3, 2500, (3, 1, 1), 128, "f32", "fused")
    f, start = _freq(128), _i32([5, 6, 7])
    all_ = A.rotate_qk(q, k, f, start=start, eps=1e-6)
    for b, i, m in ((0, 0, 1), (1, 1203, 2), (2, 2499, 1), (1, 30, 400)):
        one = A.rotate_qk(q[b:b + 1, i:i + m], k[b:b + 1, i:i + m], f, start=start[b:b + 1] + i, eps=1e-6)
        assert torch.equal(one["q"][0], all_["q"][b, i:i + m]) and torch.equal(one["k"][0], all_["k"][b, i:i + m])


def test_numbers_that_are_none(A):
    """A NaN or infinity spoils its head's row under a norm, its pair without; large numbers' squares may pass float32."""
    rng = np.random.default_rng(5)
    for dtype in ("f32", "bf16"):
        q, k = _heads(rng, 1, 4, (3, 1), 64, dtype, "dense")
        q[0, 1, 1, 3], q[0, 2, 0, 40] = float("nan"), float("inf")
        q[0, 3, 2], q[0, 0, 0], q[0, 0, 1] = q[0, 3, 2] * 1e30, 0.0, q[0, 0, 1] * 1e-30
        f = _freq(64)
        clean = np.nan_to_num(_f64(q), nan=0.0, posinf=0.0)
        for eps in (None, 1e-6):
            r = A.rotate_qk(q, k, f, start=_i32([9]), eps=eps)["q"]
            z, h = O.turned(clean, _f64(f), (9 + np.arange(4))[None, None], eps=eps)
            bad = torch.zeros_like(q, dtype=torch.bool)
            if eps is None:
                bad[0, 1, 1, [3, 35]] = bad[0, 2, 0, [8, 40]] = True
                assert not torch.isfinite(r[bad]).any()
            else:
                bad[0, 1, 1] = bad[0, 2, 0] = True
                assert torch.isnan(r[0, 1, 1]).all() and not torch.isfinite(r[0, 2, 0, [8, 40]]).any()
                assert not r[0, 2, 0, [c for c in range(64) if c not in (8, 40)]].any()
            keep = ~bad.cpu().numpy()
            off = np.abs(_f64(r) - z)[keep]
            # (numbers of 1e-30 are below float32's smallest steps times their errors: 2^-149 each)
            bound = (16 * 2.0 ** -24 * h * 1.01 + (2.0 ** -8 * np.abs(z) if dtype == "bf16" else 0) + 4 * 2.0 ** -149)[keep]
            assert (off <= bound).all()


# -- into the cache -----------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,n,Hq,H,quarters,axes,inter,weights,lay", CASES)
def test_the_cache_holds_the_64_bit_codes(A, dtype, D, B, n, Hq, H, quarters, axes, inter, weights, lay):
    rng = np.random.default_rng(D + n + Hq + 1)
    R, S = quarters * D // 4, n + 20
    q, k, v = _heads(rng, B, n, (Hq, H, H), D, dtype, lay)
    f = _freq(R, 500000.0)
    eps = None if weights == "off" else 1e-6
    qw, kw = (None, None) if weights == "off" else (_weights(rng, weights, Hq, D, dtype), _weights(rng, weights, H, D, dtype))
    cache = A.kv4_cache(2, B, H, S, D)
    cache.fill_(0xAB)
    start, base = rng.integers(0, S - n + 1, B), rng.integers(0, 100000, B)
    turn = dict(q_weight=qw, k_weight=kw, eps=eps, interleaved=inter, scale=1.0 if n % 2 else 0.83)
    if axes == 1:
        pos, ax = (base[:, None] + start[:, None] + np.arange(n))[None], None
        r = A.kv4_append_rotated(cache, 1, q, k, v, _i32(start), f, base=_i32(base), **turn)
    else:
        pos, ax = rng.integers(0, 1 << 18, (axes, B, n)), rng.integers(0, axes, R // 2)
        r = A.kv4_append_rotated(cache, 1, q, k, v, _i32(start), f, positions=_i32(pos), axes=_i32(ax), **turn)
    z, h = O.turned(_f64(q), _f64(f), pos, ax, None if qw is None else _f64(qw), eps, inter, turn["scale"])
    _close(r["q"], z, h, dtype)
    z, _ = O.turned(_f64(k), _f64(f), pos, ax, None if kw is None else _f64(kw), eps, inter, turn["scale"])
    back = A.kv4_read(cache, 1, _i32(start), n, dtype=torch.float32)
    np.testing.assert_array_equal(_f64(back["k"]), O.held(z))
    np.testing.assert_array_equal(_f64(back["v"]), O.held(_f64(v)))
    assert not r["status"].any()
    outside = torch.ones(B, S, dtype=torch.bool)
    for b in range(B):
        outside[b, start[b]:start[b] + n] = False
    assert (cache[:2] == 0xAB).all() and (cache[2:].permute(1, 3, 0, 2, 4)[outside.cuda()] == 0xAB).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("inter", [False, True])
def test_codes_on_borders(A, D, inter):
    """Quotients on halves, steps between two, largest numbers of both signs, zeros and ranges of sizes: all in
    what the first position, which turns nothing, writes; then the same turned."""
    rng = np.random.default_rng(D)
    n, H = 600, 2
    x = rng.integers(-32, 33, (1, n, 2 * H, D)) / 4.0 * np.exp2(rng.integers(-70, 18, (1, n, 2 * H, 1)))
    g = x.reshape(1, n, 2 * H, 8, D // 8)
    kind = rng.integers(0, 8, g.shape[:-1])
    g[kind == 0] = 0.0
    g[kind == 1] *= 2.0 ** -80                     # some below what a group holds
    g[kind == 2] = np.sign(g[kind == 2])
    g[kind == 3] *= 1 + 2.0 ** -23                 # beside the halves
    kv = torch.from_numpy(x.astype(np.float32)).cuda()
    q, f = torch.zeros(1, n, 1, D, device="cuda"), _freq(D)
    for pos in (np.zeros(n, int), np.arange(n)):
        cache = A.kv4_cache(1, 1, H, n, D)
        r = A.kv4_append_rotated(cache, 0, q, kv[:, :, :H], kv[:, :, H:], _i32([0]), f, positions=_i32(pos[None]), interleaved=inter)
        back = A.kv4_read(cache, 0, _i32([0]), n, dtype=torch.float32)
        z, _ = O.turned(_f64(kv[:, :, :H]), _f64(f), pos[None, None], interleaved=inter)
        np.testing.assert_array_equal(_f64(back["k"]), O.held(z))
        np.testing.assert_array_equal(_f64(back["v"]), O.held(_f64(kv[:, :, H:])))
        assert not r["status"].any()


def test_places_padding_and_bad_numbers(A):
    rng = np.random.default_rng(6)
    B, n, Hq, H, D, S = 3, 5, 3, 2, 64, 12
    for dtype in ("f32", "bf16"):
        q, k, v = _heads(rng, B, n, (Hq, H, H), D, dtype, "dense")
        k[0, 1, 1, 3], v[0, 3, 0, 9], k[1, 2, 0, 60] = float("nan"), float("inf"), -float("inf")
        cache = A.kv4_cache(1, B, H, S, D)
        start, count = [2, 9, -2], _i32([4, 5, 5])
        f = _freq(32)
        r = A.kv4_append_rotated(cache, 0, q, k, v, _i32(start), f, count=count)
        R, N = A.ROW_RANGE, A.ROW_NONFINITE
        np.testing.assert_array_equal(r["status"].cpu().numpy(), [[0, N, 0, N, 0], [0, 0, N, R, R], [R, R, 0, 0, 0]])
        rows = cache.cpu().numpy()
        assert not rows[:, 0, :, 6:].any() and not rows[:, 0, :, :2].any()        # the padding token too
        z, h = O.turned(_f64(q), _f64(f), (np.array(start)[:, None] + np.arange(n))[None])
        _close(r["q"], z, h, dtype)                                                # every token's
        back = A.kv4_read(cache, 0, _i32(start), n, dtype=torch.float32)
        kz, _ = O.turned(np.nan_to_num(_f64(k), nan=0.0, neginf=0.0), _f64(f), (np.array(start)[:, None] + np.arange(n))[None])
        clean = np.ones((B, n, H), bool)
        clean[0, 1, 1] = clean[1, 2, 0] = clean[0, 4] = clean[1, 3:] = clean[2, :2] = False
        np.testing.assert_array_equal(_f64(back["k"])[clean], O.held(kz)[clean])
        assert not back["k"][0, 1, 1, [3, 19]].any()                              # NaN: zeros
        vz = O.held(np.nan_to_num(_f64(v), posinf=O.CAP))
        np.testing.assert_array_equal(_f64(back["v"])[0, :4], vz[0, :4])


def test_graphs_and_other_streams(A):
    rng = np.random.default_rng(7)
    q, k, v = _heads(rng, 2, 3, (4, 2, 2), 128, "bf16", "fused")
    f, start = _freq(128), _i32([1, 5])
    cache, other = A.kv4_cache(1, 2, 2, 16, 128), A.kv4_cache(1, 2, 2, 16, 128)
    out = dict(q=torch.empty(2, 3, 4, 128, device="cuda", dtype=torch.bfloat16), status=torch.empty(2, 3, device="cuda", dtype=torch.int32))
    A.kv4_append_rotated(cache, 0, q, k, v, start, f, eps=1e-6, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        A.kv4_append_rotated(cache, 0, q, k, v, start, f, eps=1e-6, out=out)
        r = A.rotate_qk(q, k, f, start=start, eps=1e-6)
    q.mul_(0.5).add_(1.0)
    k.add_(0.25)
    start.add_(2)
    g.replay()
    want = A.kv4_append_rotated(other, 0, q, k, v, start, f, eps=1e-6)
    torch.cuda.synchronize()
    assert torch.equal(out["q"], want["q"]) and torch.equal(r["q"], want["q"])
    a, b = (A.kv4_read(c, 0, start, 3) for c in (cache, other))
    assert torch.equal(a["k"], b["k"]) and torch.equal(a["v"], b["v"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        q.mul_(2.0)
        mine = A.rotate_qk(q, k, f, start=start, eps=1e-6)
    s.synchronize()
    assert torch.equal(mine["q"], A.rotate_qk(q, k, f, start=start, eps=1e-6)["q"])


def test_the_binding_refuses(A):
    x = torch.zeros(2, 3, 4, 64, device="cuda")
    k, f, at = x[:, :, :2], torch.zeros(32, device="cuda"), _i32([0, 0])
    cache = A.kv4_cache(1, 2, 2, 8, 64)
    bad = [(dict(start=None), "start"), (dict(start=at.long()), "start"), (dict(inv_freq=f.double()), "inv_freq"), (dict(inv_freq=f[:, None]), "inv_freq"),
           (dict(inv_freq=torch.zeros(64, device="cuda")), "inv_freq"), (dict(k=k.bfloat16()), "k"), (dict(k=k[:1]), "k"), (dict(k=k[..., :32]), "k"),
           (dict(q=x.transpose(2, 3)), "dense"), (dict(q=x.half()), "q"), (dict(q=x[0]), "q"), (dict(positions=torch.zeros(5, 2, 3, device="cuda", dtype=torch.int32), axes=_i32([0] * 32)), "axes"),
           (dict(positions=torch.zeros(2, 2, 3, device="cuda", dtype=torch.int32)), "axes"), (dict(axes=_i32([0] * 31)), "axes"),
           (dict(positions=torch.zeros(2, 3, device="cuda", dtype=torch.int32), depth=_i32([0, 0, 0])), "positions"),
           (dict(q_weight=torch.ones(64, device="cuda")), "eps"), (dict(eps=1e-6, q_weight=torch.ones(2, 64, device="cuda")), "q_weight"),
           (dict(eps=1e-6, k_weight=torch.ones(64, device="cuda").half()), "k_weight"), (dict(depth=_i32([0, 0])), "depth"),
           (dict(out=dict(q=x.bfloat16())), "q of out"), (dict(out=dict(k=x)), "k of out")]
    for kw, match in bad:
        with pytest.raises(ValueError, match=match):
            A.rotate_qk(**{**dict(q=x, k=k, inv_freq=f, start=at), **kw})
    for kw in (dict(eps="x"), dict(scale="x")):
        with pytest.raises(TypeError):
            A.rotate_qk(x, k, f, start=at, **kw)
    for kw in (dict(eps=0.0), dict(scale=0.0), dict(inv_freq=torch.zeros(4, device="cuda"))):
        with pytest.raises(A.AcespecError):
            A.rotate_qk(**{**dict(q=x, k=k, inv_freq=f, start=at), **kw})
    good = dict(cache=cache, layer=0, q=x, k=k, v=k, start=at, inv_freq=f)
    A.kv4_append_rotated(**good)
    for kw, match in [(dict(v=x), "v"), (dict(k=x), "k"), (dict(start=None), "start"), (dict(count=at[:1]), "count"), (dict(q=x[:1]), "q"),
                      (dict(out=dict(status=at)), "status"), (dict(base=at[:1]), "base")]:
        with pytest.raises(ValueError, match=match):
            A.kv4_append_rotated(**{**good, **kw})
    with pytest.raises(A.AcespecError):
        A.kv4_append_rotated(**{**good, "layer": 1})


def test_another_device_is_refused(A, monkeypatch):
    x = torch.zeros(1, 1, 1, 64, device="cuda")
    cache, f, at = A.kv4_cache(1, 1, 1, 8, 64), torch.zeros(32, device="cuda"), _i32([0])
    monkeypatch.setattr(A, "_current_device", lambda: 1)     # as if another GPU were the current one
    for call in (lambda: A.rotate_qk(x, x, f, start=at), lambda: A.kv4_append_rotated(cache, 0, x, x, x, at, f)):
        with pytest.raises(ValueError, match="current device"):
            call()
