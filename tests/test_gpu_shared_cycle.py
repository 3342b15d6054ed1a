"""Rotation, write and attention together, as examples/edge_shared.py runs them: against the
same requests with a cache each that holds the system prompt too."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import kv4 as O  # noqa: E402
from oracle import turn as T  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("edge_shared", os.path.join(ROOT, "examples", "edge_shared.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("sizes", [dict(), dict(B=20, system=700, Hq=12, H=4, D=128, F=(3, 2, 1), branch_len=1)])
def test_a_cache_each_holds_the_same_rows(example, sizes):
    """One layer, whose inputs are the same: rows bit for bit, wherever they lie."""
    A = example.A
    r = example.step(layers=1, **sizes)
    system = r["words"].shape[1]
    B, prompt, _ = r["prompts"].shape
    own, n = r["count"], r["token"].shape[1]
    H, S, R = r["cache"].shape[2:]
    whole = A.kv4_cache(1, B, H, system + S, 2 * (R - 16))
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    at = zero + system
    m = r["model"]
    for b in range(B):      # (one at a time: a row of a matrix product may hang on how many rows there are)
        one = A.kv4_cache(1, 1, H, system, 2 * (R - 16))
        example.forward(m, r["words"], one, zero[:1])
        whole[:, b:b + 1, :, :system] = one
        assert torch.equal(one, r["shared"][:, :, :, :system])
    example.forward(m, r["prompts"], whole, at, count=own)
    tree = example.forward(m, r["drafts"], whole, at + own, mask=r["mask"], depth=r["depth"])
    last = example.forward(m, r["token"], whole, at + own)
    for b in range(B):
        top = int(own[b]) + n
        assert torch.equal(whole[:, b, :, system:system + top], r["cache"][:, b, :, :top])
        assert torch.equal(whole[:, b, :, system + top:system + int(own[b]) + len(r["depth"])], r["cache"][:, b, :, top:int(own[b]) + len(r["depth"])])
    # Attention results of values of up to 5 standard deviations differ by weights' and
    # results' 2^-8 in each of the two computations; the projection adds Hq D of them with
    # weights of variance 1 / (Hq D), a root mean square of 4 * 2^-8 * 5 at most; its own
    # bfloat16 result and the sum's, of numbers up to 8, 2 * 2^-8 * 8.
    for a, b in ((tree, r["tree"]), (last, r["last"])):
        off = (a.float() - b.float())
        assert off.square().mean().sqrt() <= 4 * 2.0 ** -8 * 5 and off.abs().max() <= 6 * 4 * 2.0 ** -8 * 5 + 2 * 2.0 ** -8 * 8


def test_the_last_token_in_float64(example):
    """Its turn from the projection's numbers, its row in the cache and its attention over both caches."""
    r = example.step(layers=1, seed=3)
    layer, system = r["model"][0], r["words"].shape[1]
    B, own = len(r["count"]), r["count"].cpu().numpy()
    p = (r["token"] @ layer.qkv).view(B, 1, -1, layer.D)
    f = layer.inv_freq.double().cpu().numpy()
    pos = (system + own)[None, :, None]
    w = {key: v.double().cpu().numpy() for key, v in layer.norms.items() if key != "eps"}
    q64, _ = T.turned(p[:, :, :layer.Hq].double().cpu().numpy(), f, pos, None, w["q_weight"], 1e-6)
    k64, _ = T.turned(p[:, :, layer.Hq:layer.Hq + layer.H].double().cpu().numpy(), f, pos, None, w["k_weight"], 1e-6)
    rows = O.values_of(r["cache"].cpu().numpy())
    prefix = O.values_of(r["shared"][:, 0].cpu().numpy())
    G = layer.Hq // layer.H
    out = np.zeros((B, layer.Hq, layer.D))
    room = np.zeros((B, layer.Hq, layer.D))
    for b in range(B):
        np.testing.assert_array_equal(rows[0, b, :, own[b]], T.held(k64[b, 0]))
        for h in range(layer.Hq):
            K, V = (np.concatenate([prefix[x, h // G, :system], rows[x, b, h // G, :own[b] + 1]]) for x in (0, 1))
            o, _, mag, M = O.attend(q64[b, :, h], K, V, np.ones((1, len(K)), bool), layer.D ** -0.5)
            out[b, h] = o[0]
            # the query's rounding to bfloat16 (2^-8 of a score's terms, twice that in a weight) and the
            # attention's own bounds (test_gpu_kv4.py)
            room[b, h] = (2 * 2.0 ** -8 * M[0] + 2.0 ** -7 + 2.0 ** -17 + 4 * 2.0 ** -20 * (M[0] + 1)) * mag[0]
    W = layer.out.double().cpu().numpy()
    x = r["token"].double().cpu().numpy()[:, 0]
    want = x + out.reshape(B, -1) @ W
    bound = room.reshape(B, -1) @ np.abs(W) + 2.0 ** -8 * (np.abs(out.reshape(B, -1) @ W) + 1e-3) + 2.0 ** -8 * np.abs(want) + 2.0 ** -8
    assert (np.abs(r["last"].double().cpu().numpy()[:, 0] - want) <= bound).all()


def test_the_least_sizes_run(example):
    r = example.step(B=2, system=20, prompt=9)
    assert torch.isfinite(r["tree"]).all() and torch.isfinite(r["last"]).all()
