"""A batch of requests behind one system prompt, over 4-bit KV caches.

The system prompt's rows are written once, into a cache of one sequence.  Each request's own
prompt, its draft tree and its next token go into the request's own cache; queries and keys
are normed and turned by their positions on the way, which start behind the system prompt,
and attend to both caches; a shared part that is long enough for its number of requests is read
once for all of them (the default sizes are not: each request reads it).  A toy model of a few
layers (random projections) stands where the draft model would.

    python examples/edge_shared.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_02514_gb300 as A  # noqa: E402


class Layer:
    def __init__(self, gen, width, Hq, H, D):
        self.Hq, self.H, self.D = Hq, H, D
        self.qkv = torch.randn(width, (Hq + 2 * H) * D, generator=gen, device="cuda").bfloat16() * width ** -0.5
        self.out = torch.randn(Hq * D, width, generator=gen, device="cuda").bfloat16() * (Hq * D) ** -0.5
        self.norms = dict(q_weight=1 + 0.1 * torch.randn(D, generator=gen, device="cuda").bfloat16(),
                          k_weight=1 + 0.1 * torch.randn(D, generator=gen, device="cuda").bfloat16(), eps=1e-6)
        self.inv_freq = 10000.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))

    def __call__(self, x, cache, layer, start, shared=None, shared_len=None, base=None, mask=None, depth=None, count=None):
        """x [B, n, width] -> x plus the layer's attention; its keys and values go into the cache."""
        B, n, _ = x.shape
        p = (x @ self.qkv).view(B, n, self.Hq + 2 * self.H, self.D)
        q, k, v = p.split([self.Hq, self.H, self.H], dim=2)        # views: nothing is copied
        q = A.kv4_append_rotated(cache, layer, q, k, v, start, self.inv_freq, base=base, depth=depth, count=count, **self.norms)["q"]
        seen = dict(mask=mask, depth=depth, count=count)
        if shared is None:
            r = A.kv4_attention(q, cache, layer, start, **seen)
        else:
            r = A.kv4_shared_attention(q, shared, shared_len, cache, layer, start, **seen)
        return x + r["out"].flatten(2) @ self.out


def forward(layers, x, cache, start, **how):
    for i, layer in enumerate(layers):
        x = layer(x, cache, i, start, **how)
    return x


def step(B=5, system=300, prompt=40, F=(2, 1, 1), branch_len=2, V=1000, width=256, Hq=8, H=2, D=64, layers=2, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    model = [Layer(gen, width, Hq, H, D) for _ in range(layers)]
    embed = torch.randn(V, width, generator=gen, device="cuda").bfloat16()
    text = lambda *shape: embed[torch.randint(V, shape, generator=gen, device="cuda")]  # noqa: E731

    # the system prompt, once
    shared, shared_len = A.kv4_cache(layers, 1, H, system + 8, D), torch.tensor([system], dtype=torch.int32, device="cuda")
    words = text(1, system)
    forward(model, words, shared, torch.zeros_like(shared_len))

    # the requests' own prompts, of different lengths
    mask, depth = A.tree_mask(F, branch_len)
    cache = A.kv4_cache(layers, B, H, prompt + len(depth) + 8, D)
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    behind = dict(shared=shared, shared_len=shared_len, base=shared_len.expand(B).contiguous())
    count = torch.tensor([prompt - 7 * b % prompt for b in range(B)], dtype=torch.int32, device="cuda")
    prompts = text(B, prompt)
    forward(model, prompts, cache, start, count=count, **behind)

    # the packed forward of their draft trees, then of one token each in the trees' place
    drafts, token = text(B, len(depth)), text(B, 1)
    tree = forward(model, drafts, cache, count, mask=mask, depth=depth, **behind)
    last = forward(model, token, cache, count, **behind)
    return dict(model=model, shared=shared, cache=cache, count=count, words=words, prompts=prompts, drafts=drafts, token=token, mask=mask,
                depth=depth, tree=tree, last=last)


if __name__ == "__main__":
    r = step()
    torch.cuda.synchronize()
    for b in range(len(r["count"])):
        print(f"request {b}: {r['words'].shape[1]} shared and {int(r['count'][b])} own positions, next state's norm {r['last'][b].float().norm():.3f}")
