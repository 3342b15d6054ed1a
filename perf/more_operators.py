"""Timed cases of the rotation of queries and keys, their write into the 4-bit KV cache, and the attention of a
batch that shares a prefix.

A case names the call (`op`) and its sizes:

  rotate   rotate_qk(): per-head norms of queries and keys and the rotation by their positions
  append   kv4_append_rotated() and kv4_read(): the same with keys and values going into the 4-bit cache, and what
           the cache then holds
  shared   kv4_shared_attention(): new tokens of a batch against a prefix that they share and against what each has
           cached itself

A cache is [2 * layers, B, H, S, D / 2 + 16] bytes.  A row is D / 8 words of eight 4-bit codes and eight bfloat16
numbers t, one for each D / 8 channels, whose step is t * 2^16: value = (code - 8) * t * 2^16.
"""
import math

import torch

own = False

DEV = "cuda"
CAP = 15.5 * 65536.0        # largest magnitude that a row holds
TINY = 2.0 ** -90           # a group whose magnitudes are all below this is stored as zeros
EPS = 1e-6


def _turn(name, op, B, n, Hq, H, D, dtype, lo, hi, R=0, axes=1, norm=True, interleaved=False, tree=0, width=40):
    return dict(name=name, op=op, B=B, n=n, Hq=Hq, H=H, D=D, dtype=dtype, lo=lo, hi=hi, R=R or D, axes=axes, norm=norm,
                interleaved=interleaved, tree=tree, width=width)


def _shared(name, B, groups, n, Hq, H, D, dtype, shared, lo, hi, window=0, sinks=0, tree=0, ragged=False):
    return dict(name=name, op="shared", B=B, groups=groups, n=n, Hq=Hq, H=H, D=D, dtype=dtype, shared=shared, lo=lo, hi=hi,
                window=window, sinks=sinks, tree=tree, ragged=ragged)


def listed():
    return [
        # one request, one new token: latency
        _turn("rotate_token_b1", "rotate", 1, 1, 32, 8, 128, "bf16", 1000, 1000),
        # image and text tokens of a float32 model, half of the channels turned by neighbouring pairs, odd lengths
        _turn("rotate_image_f32", "rotate", 3, 1537, 12, 4, 64, "f32", 0, 700, R=32, axes=3, norm=False, interleaved=True, width=37),
        # long prompts with positions of three axes
        _turn("rotate_prompt_b2", "rotate", 2, 8192, 32, 8, 128, "bf16", 0, 120000, axes=3, width=64),
        # one new token of a few requests
        _turn("append_token_b4", "append", 4, 1, 32, 8, 128, "bf16", 200, 4000),
        # the packed draft trees of a batch (16 main tokens and 64 branches)
        _turn("append_tree_b64", "append", 64, 80, 32, 8, 128, "bf16", 200, 4000, tree=16),
        # prompts of an odd length from a float32 model without norms
        _turn("append_prompt_f32", "append", 3, 4099, 12, 4, 64, "f32", 0, 700, norm=False),
        # a few requests behind a short system prompt, one new token each: latency
        _shared("shared_token_b4", 4, 1, 1, 32, 8, 128, "bf16", 2000, 10, 300),
        # a batch of requests behind a long system prompt
        _shared("shared_token_b64", 64, 1, 1, 32, 8, 128, "bf16", 16384, 100, 2000),
        # one very long document, questions of many requests
        _shared("shared_token_long", 32, 1, 1, 32, 8, 128, "bf16", 131071, 10, 500),
        # float32 queries, two prompts of eight requests each, a sliding window with four first tokens kept
        _shared("shared_window_f32", 16, 2, 1, 12, 4, 64, "f32", 6000, 50, 900, window=4096, sinks=4),
        # packed draft trees behind a system prompt
        _shared("shared_tree_b16", 16, 1, 80, 32, 8, 128, "bf16", 4096, 200, 1500, tree=16),
        # prompts of several requests behind a shared document
        _shared("shared_prompt_b4", 4, 1, 1500, 32, 8, 128, "bf16", 6001, 0, 333, ragged=True),
    ]


MOST_CELLS = 2 * 8192 * 40 * 128                          # numbers that a rotation handles
MOST_PAIRS = 4 * 1500 * 32 * 128 * (6001 + 750)           # heads x rows x keys x channels


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotate", "append", "shared", "shared"])
    D, dtype = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "f32"])
    H, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 8])
    if op != "shared":
        B, n = _log(rng, 1, 64), _log(rng, 1, 8192)
        tree = rng.choice([2, 4, 8, 16]) if rng.random() < 0.25 else 0
        if tree:
            n = 5 * tree
        while B > 1 and B * n * H * (G + 2) * D > MOST_CELLS // 2:
            B //= 2
        while n > 1 and not tree and B * n * H * (G + 2) * D > MOST_CELLS // 2:
            n //= 2
        return _turn("", op, B, n, H * G, H, D, dtype, rng.randint(0, 50), rng.randint(50, 100000 if op == "rotate" else 1000),
                     R=D // 4 * rng.choice([1, 2, 4, 4]), axes=1 if tree else rng.choice([1, 1, 2, 3, 4]), norm=rng.random() < 0.6,
                     interleaved=rng.random() < 0.4, tree=tree, width=rng.randint(3, 80))
    groups, per = rng.choice([1, 1, 1, 2, 3]), _log(rng, 1, 32)
    B = groups * per
    window, sinks = (0, 0) if rng.random() < 0.6 else (_log(rng, 16, 8192), rng.choice([0, 1, 4, 7]))
    kind = rng.choice(["token", "token", "tree", "prompt"])
    S0, hi, tree = _log(rng, 16, 65536), _log(rng, 1, 2000), 0
    n = 1
    if kind == "tree":
        tree = rng.choice([2, 4, 8, 16])
        n = 5 * tree
    elif kind == "prompt":
        n = _log(rng, 2, 2000)
        dtype = "bf16" if n > 50 else dtype
    most = MOST_PAIRS if dtype == "bf16" else MOST_PAIRS // 8
    while B * n * H * G * D * (S0 + hi + n) > most and S0 > 64:
        S0 //= 2
    while B * n * H * G * D * (S0 + hi + n) > most and n > 2 and not tree:
        n //= 2
    while B > groups and (B * n * H * G * D * (S0 + hi + n) > most or B * H * hi * D > 1 << 27):
        B -= groups
    return _shared("", B, groups, n, H * G, H, D, dtype, S0, hi // 3, hi, window=window, sinks=sinks, tree=tree,
                   ragged=kind == "prompt" and rng.random() < 0.5)


# -- what a case's sizes say -------------------------------------------------
def _lens(c):
    """Cached positions of every sequence: spread over [lo, hi], the last one exactly hi."""
    B = c["B"]
    return [c["lo"] + int((c["hi"] - c["lo"]) * ((b + 1) * 0.6180339887498949 % 1.0)) for b in range(B - 1)] + [c["hi"]]


def _counts(c):
    """New positions of every sequence."""
    return [c["n"] - (b * 37 % (c["n"] // 2 + 1) if c.get("ragged") else 0) for b in range(c["B"])]


def _shared_lens(c):
    """Positions of every shared prefix: the first as long as the case says, others a little shorter."""
    return [c["shared"] - g * (c["shared"] // 7) for g in range(c["groups"])]


def _tree(c):
    """Depths of a tree of `tree` main tokens with four branches each, and the tokens that every token sees."""
    K = c["tree"]
    depth, sees = list(range(K)), [list(range(i + 1)) for i in range(K)]
    for d in range(K):
        for _ in range(4):
            sees.append(list(range(d)) + [len(depth)])
            depth.append(d)
    return depth, sees


def _sections(c):
    """How many pairs of channels turn by each axis: a quarter by the first, the others share the rest."""
    pairs, A = c["R"] // 2, c["axes"]
    if A == 1:
        return [pairs]
    first = max(1, pairs // 4)
    rest = pairs - first
    sizes = [first] + [rest // (A - 1)] * (A - 1)
    sizes[-1] += pairs - sum(sizes)
    return sizes


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def work(case):
    c = case
    es, D, row = 4 if c["dtype"] == "f32" else 2, c["D"], c["D"] // 2 + 16
    if c["op"] != "shared":
        tokens = c["B"] * c["n"]
        numbers = tokens * (c["Hq"] + (2 if c["op"] == "append" else 1) * c["H"]) * D
        held = 2 * tokens * c["H"] * row if c["op"] == "append" else 0
        return dict(bytes=2 * numbers * es + held + 4 * tokens * c["axes"], flops=10 * numbers)
    pairs = rows = 0
    W, sinks = c["window"], c["sinks"]
    shared, per = _shared_lens(c), c["B"] // c["groups"]
    depth, sees = _tree(c) if c["tree"] else (None, None)
    lows = list(shared)
    for b, (P, count) in enumerate(zip(_lens(c), _counts(c))):
        S0 = shared[b // per]
        low = S0 + P
        for i in range(count):
            at = S0 + P + (depth[i] if depth else i)
            first = max(0, at - W + 1) if W else 0            # the first position inside the window
            low = min(low, first)
            pairs += max(0, S0 + P - first) + min(sinks, first, S0 + P)
            if depth:
                pairs += sum(S0 + P + depth[t] >= first or S0 + P + depth[t] < sinks for t in sees[i])
            else:
                pairs += at + 1 - max(S0 + P, first) + max(0, min(sinks, first) - S0 - P)
        lows[b // per] = min(lows[b // per], low)
        rows += P + count - max(0, low - S0) + max(0, min(sinks, low) - S0)
    rows += sum(S0 - low + min(sinks, low) for S0, low in zip(shared, lows))
    total = c["B"] * c["n"] * c["Hq"] * (2 * D * es + 4) + rows * 2 * c["H"] * row
    return dict(bytes=total, flops=4 * D * c["Hq"] * pairs)


# -- the cache's rows, in plain operations ------------------------------------
def _power(e):
    """2^e for whole numbers e in 64 bits (torch.ldexp goes through a power that may be a unit off)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _pack(x):
    """float64 [..., D] -> uint8 [..., D / 2 + 16]."""
    D = x.shape[-1]
    G = D // 8
    x = torch.where(x == x, x, 0.0).clamp(-CAP, CAP).reshape(*x.shape[:-1], 8, G)
    size = x.abs()
    top = size.amax(-1, keepdim=True)
    at = torch.where(size == top, torch.arange(G, device=x.device), G).amin(-1, keepdim=True)   # the first of the largest
    m, e = torch.frexp(x.gather(-1, at))
    s = torch.where(top < TINY, 0.0, -torch.round(m * 32.0) * _power(e - 8))                 # 5 significant bits
    r = torch.round(torch.where(s == 0.0, 0.0, x / torch.where(s == 0.0, 1.0, s))).clamp(-8.0, 7.0)
    code = (r.to(torch.int32) + 8).reshape(*x.shape[:-2], D // 8, 4, 2)
    shift = torch.tensor([[4 * j, 4 * j + 16] for j in range(4)], dtype=torch.int32, device=x.device)
    words = (code << shift).sum((-1, -2), dtype=torch.int32)
    t = (s[..., 0] / 65536.0).to(torch.bfloat16)
    return torch.cat([words.view(torch.uint8), t.contiguous().view(torch.uint8)], -1)


def _unpack(rows):
    """uint8 [..., D / 2 + 16] -> float32 [..., D]."""
    D = 2 * (rows.shape[-1] - 16)
    words = rows[..., :D // 2].contiguous().view(torch.int32)
    shift = torch.tensor([[4 * j, 4 * j + 16] for j in range(4)], dtype=torch.int32, device=rows.device)
    code = ((words[..., None, None] >> shift) & 15) - 8
    s = rows[..., D // 2:].contiguous().view(torch.bfloat16).float() * 65536.0
    return (code.reshape(*rows.shape[:-1], 8, D // 8) * s[..., None]).reshape(*rows.shape[:-1], D)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _prepare_turn(c, gen):
    B, n, Hq, H, D, R = c["B"], c["n"], c["Hq"], c["H"], c["D"], c["R"]
    # what one projection gives: queries, keys and values of a token lie side by side; some channels of the keys are
    # far larger than others
    qkv = _normal(gen, B, n, Hq + 2 * H, D)
    qkv[:, :, Hq:Hq + H] *= torch.exp(0.6 * _normal(gen, H, D))
    qkv = (1.7 * qkv).to(_dtype(c))
    state = dict(case=c, q=qkv[:, :, :Hq], k=qkv[:, :, Hq:Hq + H], v=qkv[:, :, Hq + H:], start=_ints(_lens(c)))
    state["inv_freq"] = (500000.0 ** (-torch.arange(R // 2, dtype=torch.float64, device=DEV) / (R // 2))).float()
    state["q_weight"] = state["k_weight"] = None
    if c["norm"]:
        state["q_weight"] = (1.0 + 0.2 * _normal(gen, D)).to(_dtype(c))
        state["k_weight"] = (1.0 + 0.2 * _normal(gen, D)).to(_dtype(c))
    state["depth"] = _ints(_tree(c)[0]) if c["tree"] else None
    state["positions"] = state["axes"] = None
    if c["axes"] > 1:
        # a few text tokens, then images of `width` columns and ten rows after one another: time, row, column (and a
        # fourth axis: the image)
        i = torch.arange(n, device=DEV)
        j = (i - 5).clamp(min=0)
        image, row, col = j // (10 * c["width"]), j // c["width"] % 10, j % c["width"]
        text = i.clamp(max=5)
        at = torch.stack([text + 40 * image, text + 40 * image + row, text + 40 * image + col, text + image])[:c["axes"]]
        state["positions"] = (at[:, None] + state["start"][None, :, None]).int().contiguous()
        sizes = _sections(c)
        state["axes"] = _ints([a for a in range(c["axes"]) for _ in range(sizes[a])])
    if c["op"] == "append":
        state["cache"] = torch.zeros(2, B, H, c["hi"] + n + 8, D // 2 + 16, dtype=torch.uint8, device=DEV)
    return state


def _prepare_shared(c, gen):
    B, n, Hq, H, D = c["B"], c["n"], c["Hq"], c["H"], c["D"]
    # a model's keys: some channels far larger than the others, and not centred
    size = torch.exp(0.6 * _normal(gen, H, 1, D))
    centre = size * 0.5 * _normal(gen, H, 1, D)

    def cache(B, S):
        got = torch.zeros(2, B, H, S, D // 2 + 16, dtype=torch.uint8, device=DEV)
        for b in range(B):
            got[0, b] = _pack((centre + size * _normal(gen, H, S, D)).double())
            got[1, b] = _pack(_normal(gen, H, S, D).double())
        return got

    state = dict(case=c, shared=cache(c["groups"], c["shared"]), cache=cache(B, c["hi"] + n + 8), shared_len=_ints(_shared_lens(c)),
                 prefix_len=_ints(_lens(c)))
    spread = size.reshape(H, 1, D).expand(H, Hq // H, D).reshape(Hq, D)
    state["q"] = (1.5 * _normal(gen, B, n, Hq, D) / spread).to(_dtype(c))
    state["count"] = _ints(_counts(c)) if c["ragged"] else None
    state["mask"] = state["depth"] = None
    if c["tree"]:
        depth, sees = _tree(c)
        words = [[0] * ((n + 31) // 32) for _ in range(n)]
        for row, seen in zip(words, sees):
            for t in seen:
                row[t // 32] |= 1 << (t % 32)
        flat = torch.tensor(words, dtype=torch.int64)
        state["mask"] = torch.where(flat >= 1 << 31, flat - (1 << 32), flat).to(torch.int32).to(DEV)
        state["depth"] = _ints(depth)
    return state


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (_prepare_shared if case["op"] == "shared" else _prepare_turn)(case, gen)


# -- a user's calls -------------------------------------------------------------
def _run_own(s):
    import paper_2609_02514_gb300 as A
    c = s["case"]
    if c["op"] == "shared":
        r = A.kv4_shared_attention(s["q"], s["shared"], s["shared_len"], s["cache"], 0, s["prefix_len"], mask=s["mask"],
                                   depth=s["depth"], count=s["count"], window=c["window"], sinks=c["sinks"])
        return dict(out=r["out"], lse=r["lse"])
    turn = dict(depth=s["depth"], positions=s["positions"], axes=s["axes"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                eps=EPS if c["norm"] else None, interleaved=c["interleaved"])
    if c["op"] == "rotate":
        r = A.rotate_qk(s["q"], s["k"], s["inv_freq"], start=s["start"], **turn)
        return dict(q=r["q"], k=r["k"])
    r = A.kv4_append_rotated(s["cache"], 0, s["q"], s["k"], s["v"], s["start"], s["inv_freq"], **turn)
    back = A.kv4_read(s["cache"], 0, s["start"], c["n"], dtype=_dtype(c))
    return dict(q=r["q"], k=back["k"], v=back["v"], status=r["status"])


# -- the plain forms --------------------------------------------------------------
def _angles(s):
    """The angle of every token's pairs in 64 bits: [B, n, 1, R / 2]."""
    c = s["case"]
    if s["positions"] is not None:
        at = s["positions"][s["axes"].long()].permute(1, 2, 0)                                     # [B, n, R / 2]
    else:
        at = (s["start"][:, None] + (s["depth"] if s["depth"] is not None else torch.arange(c["n"], device=DEV))[None])[..., None]
    return (at.double() * s["inv_freq"].double())[:, :, None]


def _turned(s, x, weight, kind):
    """Heads of x [B, n, heads, D] normed and turned, in numbers of type `kind`."""
    c = s["case"]
    x = x.to(kind)
    if c["norm"]:
        x = x * weight.to(kind) * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)       # (equal products stay equal)
    angle = _angles(s)
    cos, sin = torch.cos(angle).to(kind), torch.sin(angle).to(kind)
    y, rest = x[..., :c["R"]], x[..., c["R"]:]
    if c["interleaved"]:
        u, v = y[..., 0::2], y[..., 1::2]
        y = torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)
    else:
        u, v = y.chunk(2, -1)
        y = torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
    return torch.cat([y, rest], -1)


def _append_plain(s):
    c = s["case"]
    B, n, H = c["B"], c["n"], c["H"]
    q = _turned(s, s["q"], s["q_weight"], torch.float32).to(_dtype(c))
    # a code may lie next to a border, where 32 bits would not tell
    new = torch.stack([_turned(s, s["k"], s["k_weight"], torch.float64), s["v"].double()])
    status = (~torch.isfinite(new)).any(-1).any(-1).any(0).to(torch.int32)
    b, h = torch.arange(B, device=DEV)[:, None, None], torch.arange(H, device=DEV)[None, None, :]
    at = (s["start"][:, None].long() + torch.arange(n, device=DEV))[:, :, None]
    s["cache"][:2, b, h, at] = _pack(new)
    k, v = _unpack(s["cache"][:2, b, h, at]).to(_dtype(c))
    return dict(q=q, k=k, v=v, status=status)


def _visible(s):
    """Which positions, the shared ones first, every query sees: [B, n, S0 + S]."""
    c = s["case"]
    n, S0, S = c["n"], s["shared"].shape[3], s["cache"].shape[3]
    base = s["shared_len"].long().repeat_interleave(c["B"] // c["groups"])[:, None, None]
    P = s["prefix_len"].long()[:, None, None]
    i = torch.arange(n, device=DEV)[None, :, None]
    count = c["n"] if s["count"] is None else s["count"].long()[:, None, None]
    slot = torch.arange(S0, device=DEV)[None, None, :]
    key = torch.arange(S, device=DEV)[None, None, :]
    t = (key - P).clamp(0, n - 1)                                     # the new token at a position
    if s["mask"] is None:
        sees, step, where = key <= P + i, i, key
    else:
        word = s["mask"][torch.arange(n, device=DEV)[None, :, None], t >> 5]
        sees = ((word >> (t & 31).int()) & 1) == 1
        depth = s["depth"].long()
        step, where = depth[None, :, None], torch.where(key >= P, P + depth[t], key)
    sees = ((key < P) | sees) & (key < P + count) & (i < count)
    first = (slot < base) & (i < count)
    if c["window"]:
        low = base + P + step - c["window"]
        sees = sees & ((base + where > low) | (base + where < c["sinks"]))
        first = first & ((slot > low) | (slot < c["sinks"]))
    return torch.cat([first.expand(c["B"], n, S0), sees.expand(c["B"], n, S)], -1)


def _shared_plain(s):
    c = s["case"]
    B, n, Hq, D = s["q"].shape
    H, G, groups = c["H"], Hq // c["H"], c["groups"]
    K0, V0 = _unpack(s["shared"][0])[:, None], _unpack(s["shared"][1])[:, None]                    # [groups, 1, H, S0, D]
    K, V = _unpack(s["cache"][0]), _unpack(s["cache"][1])                                          # [B, H, S, D]
    S0 = K0.shape[3]
    q = s["q"].float().reshape(B, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, D)
    x0 = (q.reshape(groups, -1, H, G * n, D) @ K0.transpose(-1, -2)).reshape(B, H, G, n, S0)
    x = torch.cat([x0, (q @ K.transpose(-1, -2)).reshape(B, H, G, n, -1)], -1) / math.sqrt(D)
    x = x.masked_fill(~_visible(s)[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    p = p.reshape(B, H, G * n, -1)
    o = (p[..., :S0].reshape(groups, -1, H, G * n, S0) @ V0).reshape(B, H, G * n, D) + p[..., S0:] @ V
    o = o.reshape(B, H, G, n, D) / torch.where(total == 0.0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    return dict(out=o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D).to(s["q"].dtype), lse=lse.permute(0, 3, 1, 2).reshape(B, n, Hq))


def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["case"]["op"] == "shared":
        return _shared_plain(s)
    if s["case"]["op"] == "append":
        return _append_plain(s)
    dtype = _dtype(s["case"])
    return dict(q=_turned(s, s["q"], s["q_weight"], torch.float32).to(dtype), k=_turned(s, s["k"], s["k_weight"], torch.float32).to(dtype))


# -- the same from the definitions, in 64 bits --------------------------------
def _turned64(s, x, weight):
    """Pair by pair: the product of two complex numbers."""
    c = s["case"]
    x = x.double().clone()
    if weight is not None:
        x = x * weight.double() / torch.sqrt(x.square().sum(-1, keepdim=True) / c["D"] + EPS)
    out = x.clone()
    half = c["R"] // 2
    for j in range(half):
        u, v = (2 * j, 2 * j + 1) if c["interleaved"] else (j, j + half)
        if s["positions"] is not None:
            at = s["positions"][int(s["axes"][j])].double()
        else:
            steps = s["depth"] if s["depth"] is not None else torch.arange(c["n"], device=DEV)
            at = s["start"].double()[:, None] + steps.double()
        turn = torch.polar(torch.ones_like(at), at * s["inv_freq"][j].double())[..., None]
        z = torch.complex(x[..., u], x[..., v]) * turn
        out[..., u], out[..., v] = z.real, z.imag
    return out


def _two64(e):
    """2^e, from a table."""
    return torch.tensor([2.0 ** i for i in range(-300, 301)], dtype=torch.float64, device=DEV)[(e.long() + 300).clamp(0, 600)]


def _values64(x):
    """What a row of numbers is held as."""
    D = x.shape[-1]
    g = x.double().unflatten(-1, (8, D // 8))
    size = g.abs().amax(-1, keepdim=True)
    last = torch.zeros_like(size)
    for e in reversed(range(D // 8)):                                 # the first of the largest decides the sign
        last = torch.where(g[..., e:e + 1].abs() == size, g[..., e:e + 1], last)
    m, e = torch.frexp(last)
    step = -torch.round(m * 32.0) / 32.0 * _two64(e) / 8.0
    step = torch.where(size < 2.0 ** -90, torch.zeros_like(step), step)
    n = torch.round(g / torch.where(step == 0, torch.ones_like(step), step)).clamp(-8, 7)
    return (n * step).flatten(-2)


def _held64(rows):
    """The numbers of cache rows, byte by byte."""
    half = rows.shape[-1] - 16
    D = 2 * half
    r = rows.long()
    out = torch.empty(*rows.shape[:-1], D, dtype=torch.float64, device=rows.device)
    lo, hi = r[..., half::2], r[..., half + 1::2]
    e, m = ((hi & 127) << 1) | (lo >> 7), lo & 127
    t = (1.0 + m.double() / 128.0) * _two64(e - 127 + 16) * torch.where(hi >= 128, -1.0, 1.0) * (e > 0)
    for x in range(D):
        word, j, odd = x // 8, (x % 8) // 2, x % 2
        byte = r[..., 4 * word + 2 * odd + j // 2]
        code = (byte >> (4 * (j % 2))) & 15
        out[..., x] = (code - 8).double() * t[..., x // (D // 8)]
    return out


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "rotate":
        return dict(q=_turned64(s, s["q"], s["q_weight"]), k=_turned64(s, s["k"], s["k_weight"]))
    if c["op"] == "append":
        status = torch.zeros(c["B"], c["n"], dtype=torch.int32, device=DEV)
        return dict(q=_turned64(s, s["q"], s["q_weight"]), k=_values64(_turned64(s, s["k"], s["k_weight"])), v=_values64(s["v"]),
                    status=status)
    if work(c)["flops"] > 2e12:
        return None
    B, n, Hq, H, D, W = c["B"], c["n"], c["Hq"], c["H"], c["D"], c["window"]
    G, per, lens, counts, shared = Hq // H, B // c["groups"], _lens(c), _counts(c), _shared_lens(c)
    out = torch.zeros(B, n, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, n, Hq), -math.inf, dtype=torch.float64, device=DEV)
    steps, seen = _tree(c) if c["tree"] else (list(range(n)), None)
    for g in range(c["groups"]):
        S0 = shared[g]
        for h in range(H):
            K0, V0 = _held64(s["shared"][0, g, h, :S0]), _held64(s["shared"][1, g, h, :S0])
            for b in range(g * per, (g + 1) * per):
                P, m = lens[b], counts[b]
                K = torch.cat([K0, _held64(s["cache"][0, b, h, :P + m])])
                V = torch.cat([V0, _held64(s["cache"][1, b, h, :P + m])])
                pos = S0 + P + torch.tensor(steps[:m], device=DEV)
                where = torch.cat([torch.arange(S0 + P, device=DEV), pos])
                ok = where[None, :] <= pos[:, None]
                if seen is not None:
                    sub = torch.zeros(m, m, dtype=torch.bool)
                    for i in range(m):
                        sub[i, [t for t in seen[i] if t < m]] = True
                    ok[:, :S0 + P] = True
                    ok[:, S0 + P:] = sub.to(DEV)
                if W:
                    ok &= (pos[:, None] - where[None, :] < W) | (where[None, :] < c["sinks"])
                x = torch.einsum("mgd,sd->gms", s["q"][b, :m, h * G:(h + 1) * G].double(), K) / math.sqrt(D)
                x = torch.where(ok[None], x, -math.inf)
                z = torch.logsumexp(x, -1)
                lse[b, :m, h * G:(h + 1) * G] = z.T
                w = torch.exp(x - torch.where(torch.isfinite(z), z, torch.zeros_like(z))[..., None])
                out[b, :m, h * G:(h + 1) * G] = torch.einsum("gms,sd->mgd", w, V)
    return dict(out=out, lse=lse)
