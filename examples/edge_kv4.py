"""One speculation cycle of the edge over a 4-bit KV cache.

The prompt's keys and values are quantised as they are written and attended to;
the draft tree is run in one packed forward with the tree mask; the cloud's
verdict is looked up in the branch cache; the hit branch's rows move behind the
accepted tokens.  A hit branch begins with the verdict's token, so nothing is run
again: the tree's forward has the state after it.  Elsewhere (a miss, or a chain
accepted whole) the verdict's token is run, and those sequences alone get its row.
A toy model of a few layers (random projections) stands where the draft model would.

    python examples/edge_kv4.py
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

    def __call__(self, x, cache, layer, start, count=None, **seen):
        """x [B, n, width] -> x plus the layer's attention; its keys and values go into the cache
        (those of count[b] tokens)."""
        B, n, _ = x.shape
        p = (x @ self.qkv).view(B, n, self.Hq + 2 * self.H, self.D)
        q, k, v = p.split([self.Hq, self.H, self.H], dim=2)        # views: nothing is copied
        A.kv4_append(cache, layer, k, v, start, count=count)
        return x + A.kv4_attention(q, cache, layer, start, count=count, **seen)["out"].flatten(2) @ self.out


def forward(layers, x, cache, start, **seen):
    for i, layer in enumerate(layers):
        x = layer(x, cache, i, start, **seen)
    return x


def cycle(B=4, prompt=300, K=4, F=(3, 2, 1, 1), branch_len=2, V=1000, width=256, Hq=8, H=2, D=64, depth=2, window=0, sinks=0,
          seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = K + sum(F) * branch_len
    layers = [Layer(gen, width, Hq, H, D) for _ in range(depth)]
    embed = torch.randn(V, width, generator=gen, device="cuda").bfloat16()
    cache = A.kv4_cache(depth, B, H, prompt + n + 8, D)
    seen = dict(window=window, sinks=sinks)

    # the prompt, in one piece
    tokens = torch.randint(V, (B, prompt), generator=gen, device="cuda")
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    forward(layers, embed[tokens], cache, start, **seen)
    prefix = start + prompt

    # the draft: a main chain, and at every depth the most probable other tokens
    q = torch.softmax(3 * torch.randn(B, K, V, generator=gen, device="cuda"), -1)
    chain = torch.multinomial(q.view(-1, V), 1, generator=gen).view(B, K).int()
    branches = A.cache_build(q, chain, F)["branch_tok"]
    mask, depths = A.tree_mask(F, branch_len)
    follow = torch.randint(V, (B, sum(F), branch_len - 1), generator=gen, device="cuda")
    tree = torch.cat([chain.long(), torch.cat([branches.long()[..., None], follow], -1).flatten(1)], 1)
    state = forward(layers, embed[tree], cache, prefix, mask=mask, depth=depths, **seen)

    # the cloud's verdict on the chain (target logits that agree in part)
    z = torch.log(q)
    z = torch.cat([z, z[:, -1:]], 1) + 1.5 * torch.randn(B, K + 1, V, generator=gen, device="cuda")
    u = torch.rand(B, K + 1, generator=gen, device="cuda").clamp(1e-6, 1 - 1e-6)
    verdict = A.verify(z, q, chain, u, 1.0, 0.9)
    slot = A.cache_lookup(branches, F, verdict["accept_len"], verdict["out_token"])

    # the hit branch moves behind the accepted tokens; a rejected tail is dropped
    new_len = A.compact_kv(cache, prefix, verdict["accept_len"], slot, K, branch_len)
    # what there is to run: the verdict's token, where no branch held it
    fed = (slot < 0).int()
    x = forward(layers, embed[verdict["out_token"].long()][:, None], cache, new_len, count=fed, **seen)
    last = K + slot.clamp(min=0).long() * branch_len + branch_len - 1          # a hit branch's last row in the tree
    hidden = torch.where(fed[:, None].bool(), x[:, 0], state[torch.arange(B, device="cuda"), last])[:, None]
    return dict(cache=cache, prefix=prefix, new_len=new_len, length=new_len + fed, slot=slot, accept_len=verdict["accept_len"],
                out_token=verdict["out_token"], hidden=hidden, prompt=tokens, tree=tree, embed=embed, layers=layers)


if __name__ == "__main__":
    r = cycle()
    torch.cuda.synchronize()
    for b in range(len(r["slot"])):
        print(f"sequence {b}: accepted {int(r['accept_len'][b])}, slot {int(r['slot'][b])}, "
              f"cache {int(r['prefix'][b])} -> {int(r['length'][b])}")
