"""What the example's cycle (examples/edge_kv4.py) leaves in the cache: every token of
the text once, at its position, and the tree's own rows for them, moved and not
rewritten."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
K, L, F, PROMPT = 4, 2, (3, 2, 1, 1), 300


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("edge_kv4", os.path.join(ROOT, "examples", "edge_kv4.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_cache_holds_the_text_once(example):
    """The token of a cached row is the one whose first-layer key is nearest."""
    A = example.A
    hits = others = 0
    for seed in range(8):
        r = example.cycle(seed=seed)
        layer = r["layers"][0]
        keys = (r["embed"] @ layer.qkv).float().view(-1, layer.Hq + 2 * layer.H, layer.D)[:, layer.Hq:layer.Hq + layer.H].flatten(1)
        zero = torch.zeros(len(r["slot"]), dtype=torch.int32, device="cuda")
        rows = A.kv4_read(r["cache"], 0, zero, r["cache"].shape[3], dtype=torch.float32)["k"].flatten(2)
        for b in range(len(zero)):
            al, slot = int(r["accept_len"][b]), int(r["slot"][b])
            text = r["prompt"][b].tolist() + r["tree"][b, :al].tolist()
            if slot >= 0:
                hits += 1
                branch = r["tree"][b, K + slot * L:K + (slot + 1) * L].tolist()
                assert branch[0] == int(r["out_token"][b])
                text += branch
            else:
                others += 1
                text.append(int(r["out_token"][b]))
            assert int(r["length"][b]) == len(text)
            near = torch.cdist(rows[b, :len(text)], keys).argmin(1)
            assert near.tolist() == text, (seed, b, slot)
        assert torch.isfinite(r["hidden"]).all()
    assert hits >= 3 and others >= 3


def test_the_trees_rows_are_moved(example, monkeypatch):
    before = []
    move = example.A.compact_kv
    monkeypatch.setattr(example.A, "compact_kv", lambda kv, *a, **k: (before.append(kv.clone()), move(kv, *a, **k))[1])
    for seed in range(4):
        r = example.cycle(seed=seed)
        was = before.pop()
        for b in range(len(r["slot"])):
            al, slot = int(r["accept_len"][b]), int(r["slot"][b])
            kept = PROMPT + al
            assert torch.equal(r["cache"][:, b, :, :kept], was[:, b, :, :kept])
            if slot >= 0:
                src = PROMPT + K + slot * L
                assert torch.equal(r["cache"][:, b, :, kept:kept + L], was[:, b, :, src:src + L])
