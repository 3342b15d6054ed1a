"""Timed cases of the 4-bit KV cache and the attention that reads it.

A case names the call (`op`) and its sizes:

  cache    kv4_append() and kv4_read(): new keys and values are quantised as they are written, and read back
  read     kv4_read(): a range of the cache as numbers again
  attend   kv4_attention(): single tokens, a packed draft tree or a prompt against the cache, with or
           without a sliding window and the first tokens that stay visible

The cache is [2 * layers, B, H, S, D / 2 + 16] bytes.  A row is D / 8 words of eight 4-bit codes and eight
bfloat16 numbers t, one for each D / 8 channels, whose step is t * 2^16: value = (code - 8) * t * 2^16.
"""
import math

import torch

own = False

DEV = "cuda"
CAP = 15.5 * 65536.0        # largest magnitude that a row holds
TINY = 2.0 ** -90           # a group whose magnitudes are all below this is stored as zeros


def _cache(name, B, n, H, D, dtype, lo, hi, op="cache"):
    return dict(name=name, op=op, B=B, n=n, H=H, D=D, dtype=dtype, lo=lo, hi=hi)


def _attend(name, B, n, Hq, H, D, dtype, lo, hi, form="causal", window=0, sinks=0, K=0, F0=0, decay=1.0, L=1, ragged=False):
    return dict(name=name, op="attend", B=B, n=n, Hq=Hq, H=H, D=D, dtype=dtype, lo=lo, hi=hi, form=form, window=window,
                sinks=sinks, K=K, F0=F0, decay=decay, L=L, ragged=ragged)


def listed():
    return [
        # one request, one new token: latency of the write and of the read
        _cache("cache_token_b1", 1, 1, 8, 128, "bf16", 1000, 1000),
        # the packed draft trees of a batch (16 main tokens and 64 branches) as they are written
        _cache("cache_tree_b64", 64, 80, 8, 128, "bf16", 200, 4000),
        # prompts of an odd length from a float32 model
        _cache("cache_prompt_f32", 3, 4099, 4, 64, "f32", 0, 700),
        # a short stretch of one cache, for inspection or to hand over
        _cache("read_b1_f32", 1, 257, 2, 64, "f32", 31, 31, op="read"),
        # whole caches leave their 4 bits
        _cache("read_b8", 8, 16384, 8, 128, "bf16", 0, 64, op="read"),
        # one request, one new token, a short cache: latency
        _attend("token_b1", 1, 1, 32, 8, 128, "bf16", 1000, 1000),
        # a batch of requests of very different lengths
        _attend("token_b64", 64, 1, 32, 8, 128, "bf16", 200, 8191),
        # one request with a very long cache
        _attend("token_long", 1, 1, 32, 8, 128, "bf16", 131071, 131071),
        # float32 queries, an odd group of heads, a sliding window with four first tokens kept
        _attend("token_window_f32", 16, 1, 12, 4, 64, "f32", 300, 16384, window=1024, sinks=4),
        # the packed forward of a draft tree: 16 main tokens and 64 branches
        _attend("tree_b16", 16, 80, 32, 8, 128, "bf16", 1000, 6000, form="tree", K=16, F0=4, decay=1.0),
        # prompts in one piece behind a window, every head with its own keys
        _attend("prompt_window", 4, 2048, 16, 16, 64, "bf16", 5000, 8192, window=1024, sinks=4),
        # long prompts of two requests behind what is cached already
        _attend("prompt_b2", 2, 4096, 32, 8, 128, "bf16", 3500, 4090, ragged=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["cache", "read", "token", "token", "tree", "prompt"])
    D, dtype = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "f32"])
    H = rng.choice([1, 2, 4, 8])
    if kind in ("cache", "read"):
        B, n = _log(rng, 1, 64), _log(rng, 1, 8192)
        while B * n * H * D > 8 * 8192 * 8 * 128:
            n = max(1, n // 2)
        return _cache("", B, n, H, D, dtype, rng.randint(0, 50), rng.randint(50, 1000), op=kind)
    G = rng.choice([1, 2, 3, 4, 5, 8])
    window, sinks = (0, 0) if rng.random() < 0.6 else (_log(rng, 16, 4096), rng.choice([0, 1, 4, 7]))
    if kind == "token":
        B, hi = _log(rng, 1, 64), _log(rng, 64, 65536)
        while B * hi * H * D > 64 * 8192 * 8 * 128 // 2:
            hi //= 2
        return _attend("", B, 1, H * G, H, D, dtype, max(1, hi // rng.choice([1, 4, 40])), hi, window=window, sinks=sinks)
    if kind == "tree":
        K, F0, L = rng.choice([2, 4, 8, 16]), rng.randint(1, 6), rng.choice([1, 1, 2, 3])
        c = _attend("", _log(rng, 1, 32), 0, H * G, H, D, dtype, 0, _log(rng, 64, 8192), form="tree", window=window, sinks=sinks,
                    K=K, F0=F0, decay=rng.choice([1.0, 0.9, 0.7]), L=L)
        c["lo"], c["n"] = c["hi"] // 3, _tree_tokens(c)
        return c
    n, hi = _log(rng, 2, 4096), _log(rng, 1, 8192)
    dtype = "bf16" if n > 200 else dtype
    B = _log(rng, 1, 8)
    while B > 1 and B * n * H * G * (hi + n) > 2 * 2000 * 32 * 6000:
        B //= 2
    while n > 2 and B * n * H * G * (hi + n) > 2 * 2000 * 32 * 6000:
        n //= 2
    return _attend("", B, n, H * G, H, D, dtype, hi // 2, hi, window=window, sinks=sinks, ragged=rng.random() < 0.5)


# -- what a case's sizes say -------------------------------------------------
def _lens(c):
    """Cached positions of every sequence: spread over [lo, hi], the last one exactly hi."""
    B = c["B"]
    return [c["lo"] + int((c["hi"] - c["lo"]) * ((b + 1) * 0.6180339887498949 % 1.0)) for b in range(B - 1)] + [c["hi"]]


def _counts(c):
    """New positions of every sequence."""
    return [c["n"] - (b * 37 % (c["n"] // 2 + 1) if c.get("ragged") else 0) for b in range(c["B"])]


def _fans(c):
    return [max(0, int(round(c["F0"] * c["decay"] ** d))) for d in range(c["K"])]


def _tree_tokens(c):
    return c["K"] + sum(_fans(c)) * c["L"]


def _tree(c):
    """Lists of the tree's depths and of the tokens that every token sees: the main chain, then the branches in order."""
    K, L = c["K"], c["L"]
    depth, sees = list(range(K)), [list(range(q + 1)) for q in range(K)]
    for d, f in enumerate(_fans(c)):
        for _ in range(f):
            first = len(depth)
            for o in range(L):
                depth.append(d + o)
                sees.append(list(range(d)) + list(range(first, first + o + 1)))
    return depth, sees


def _capacity(c):
    return c["hi"] + c["n"] + 8


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def work(case):
    c = case
    es, D, row = 4 if c["dtype"] == "f32" else 2, c["D"], c["D"] // 2 + 16
    if c["op"] != "attend":
        cells = 2 * c["B"] * c["n"] * c["H"]
        return dict(bytes=cells * (D * es * (2 if c["op"] == "cache" else 1) + row), flops=cells * D * 4)
    G_rows = c["n"] * c["Hq"]
    pairs = rows = 0
    depth, sees = _tree(c) if c["form"] == "tree" else (None, None)
    W, sinks = c["window"], c["sinks"]
    for P, count in zip(_lens(c), _counts(c)):
        low = P
        for i in range(count):
            at = P + (depth[i] if depth else i)
            first = max(0, at - W + 1) if W else 0       # the first position inside the window
            low = min(low, first)
            pairs += max(0, P - first) + min(sinks, first, P)
            if depth:
                pairs += sum(P + depth[t] >= first or P + depth[t] < sinks for t in sees[i])
            else:
                pairs += at + 1 - max(P, first) + max(0, min(sinks, first) - P)
        rows += P + count - low + min(sinks, low)
    total = c["B"] * G_rows * (2 * D * es + 4) + rows * 2 * c["H"] * row
    return dict(bytes=total, flops=4 * D * c["Hq"] * pairs)


# -- the cache's rows, in plain operations ------------------------------------
def _pack(x):
    """float32 [..., D] -> uint8 [..., D / 2 + 16]."""
    D = x.shape[-1]
    G = D // 8
    x = torch.where(x == x, x, 0.0).clamp(-CAP, CAP).reshape(*x.shape[:-1], 8, G)
    size = x.abs()
    top = size.amax(-1, keepdim=True)
    at = torch.where(size == top, torch.arange(G, device=x.device), G).amin(-1, keepdim=True)   # the first of the largest
    a = torch.where(top < TINY, 0.0, -x.gather(-1, at) * 2.0 ** -19).contiguous()
    bits = a.view(torch.int32)
    mag = bits & 0x7FFFFFFF
    t = (((mag + 0x3FFFF + ((mag >> 19) & 1)) & ~0x7FFFF) | (bits & -0x80000000)).view(torch.float32)   # 5 significant bits
    s = t * 65536.0
    r = torch.where(s == 0.0, 0.0, torch.round(x / torch.where(s == 0.0, 1.0, s)))
    d = x - r * s                                     # exact; a quotient rounded onto a half is set right by it
    r = (r + torch.where(d.abs() > 0.5 * s.abs(), torch.sign(d) * torch.sign(s), 0.0)).clamp(-8.0, 7.0)
    code = (r.to(torch.int32) + 8).reshape(*x.shape[:-2], D // 8, 4, 2)
    shift = torch.tensor([[4 * j, 4 * j + 16] for j in range(4)], dtype=torch.int32, device=x.device)
    words = (code << shift).sum((-1, -2), dtype=torch.int32)
    return torch.cat([words.view(torch.uint8), t[..., 0].to(torch.bfloat16).contiguous().view(torch.uint8)], -1)


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


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV).manual_seed(seed)
    B, n, H, D, S = c["B"], c["n"], c["H"], c["D"], _capacity(c)
    Hq = c.get("Hq", H)
    # a model's keys: some channels far larger than the others, and not centred
    size = torch.exp(0.6 * _normal(gen, H, 1, D))
    centre = size * 0.5 * _normal(gen, H, 1, D)
    start = torch.tensor(_lens(c), dtype=torch.int32, device=DEV)
    state = dict(case=c, start=start, layer=0)
    cache = torch.zeros(2, B, H, S, D // 2 + 16, dtype=torch.uint8, device=DEV)
    if c["op"] != "cache":
        for b in range(B):
            cache[0, b] = _pack((centre + size * _normal(gen, H, S, D)).bfloat16().float())
            cache[1, b] = _pack(_normal(gen, H, S, D).bfloat16().float())
    state["cache"] = cache
    if c["op"] == "cache":
        # what one projection gives: queries, keys and values of a token lie side by side
        qkv = _normal(gen, B, n, 3 * H, D)
        qkv[:, :, H:2 * H] = qkv[:, :, H:2 * H] * size[:, 0] + centre[:, 0]
        qkv = qkv.to(_dtype(c))
        state.update(k=qkv[:, :, H:2 * H], v=qkv[:, :, 2 * H:])
    if c["op"] == "attend":
        spread = size.reshape(H, 1, D).expand(H, Hq // H, D).reshape(Hq, D)
        state["q"] = (1.5 * _normal(gen, B, n, Hq, D) / spread).to(_dtype(c))
        state["count"] = torch.tensor(_counts(c), dtype=torch.int32, device=DEV) if c["ragged"] else None
        state["mask"] = state["depth"] = None
        if c["form"] == "tree":
            depth, sees = _tree(c)
            words = [[0] * ((n + 31) // 32) for _ in range(n)]
            for row, seen in zip(words, sees):
                for t in seen:
                    row[t // 32] |= 1 << (t % 32)
            flat = torch.tensor(words, dtype=torch.int64)
            state["mask"] = torch.where(flat >= 1 << 31, flat - (1 << 32), flat).to(torch.int32).to(DEV)
            state["depth"] = torch.tensor(depth, dtype=torch.int32, device=DEV)
    return state


def _run_own(s):
    import paper_2609_02514_gb300 as A
    c = s["case"]
    if c["op"] == "cache":
        status = A.kv4_append(s["cache"], s["layer"], s["k"], s["v"], s["start"])
        back = A.kv4_read(s["cache"], s["layer"], s["start"], c["n"], dtype=_dtype(c))
        return dict(k=back["k"], v=back["v"], status=status)
    if c["op"] == "read":
        back = A.kv4_read(s["cache"], s["layer"], s["start"], c["n"], dtype=_dtype(c))
        return dict(k=back["k"], v=back["v"])
    r = A.kv4_attention(s["q"], s["cache"], s["layer"], s["start"], mask=s["mask"], depth=s["depth"], count=s["count"],
                        window=c["window"], sinks=c["sinks"])
    return dict(out=r["out"], lse=r["lse"])


def _rows_at(s):
    """Indices of the cells that the case's new positions take: [B, 1], [H], [B, n]."""
    c = s["case"]
    at = s["start"][:, None].long() + torch.arange(c["n"], device=DEV)
    return torch.arange(c["B"], device=DEV)[:, None, None], torch.arange(c["H"], device=DEV)[None, None, :], at[:, :, None]


def _read_plain(s):
    b, h, at = _rows_at(s)
    planes = s["cache"][2 * s["layer"]:2 * s["layer"] + 2]
    return _unpack(planes[:, b, h, at]).to(_dtype(s["case"]))


def _visible(s):
    """Which cached positions every query sees: [B, n, S]."""
    c = s["case"]
    n, S = c["n"], s["cache"].shape[3]
    P = s["start"].long()[:, None, None]
    key = torch.arange(S, device=DEV)[None, None, :]
    i = torch.arange(n, device=DEV)[None, :, None]
    t = (key - P).clamp(0, n - 1)                                     # the new token at a position
    if s["mask"] is None:
        sees, where_q, where_k = key <= P + i, P + i, key
    else:
        word = s["mask"][torch.arange(n, device=DEV)[None, :, None], t >> 5]
        sees = ((word >> (t & 31).int()) & 1) == 1
        depth = s["depth"].long()
        where_q, where_k = P + depth[None, :, None], torch.where(key >= P, P + depth[t], key)
    count = c["n"] if s["count"] is None else s["count"].long()[:, None, None]
    sees = ((key < P) | sees) & (key < P + count) & (i < count)
    if c["window"]:
        sees = sees & ((where_k > where_q - c["window"]) | (where_k < c["sinks"]))
    return sees


def _attend_plain(s):
    c = s["case"]
    B, n, Hq, D = s["q"].shape
    H, G = c["H"], Hq // c["H"]
    K, V = _unpack(s["cache"][2 * s["layer"]]), _unpack(s["cache"][2 * s["layer"] + 1])       # [B, H, S, D]
    q = s["q"].float().reshape(B, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, D)
    x = (q @ K.transpose(-1, -2)).reshape(B, H, G, n, -1) / math.sqrt(D)
    x = x.masked_fill(~_visible(s)[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = (p.reshape(B, H, G * n, -1) @ V).reshape(B, H, G, n, D) / torch.where(total == 0.0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    return dict(out=o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D).to(s["q"].dtype), lse=lse.permute(0, 3, 1, 2).reshape(B, n, Hq))


def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["case"]["op"] == "attend":
        return _attend_plain(s)
    if s["case"]["op"] == "read":
        k, v = _read_plain(s)
        return dict(k=k, v=v)
    b, h, at = _rows_at(s)
    new = torch.stack([s["k"], s["v"]]).float()
    s["cache"][2 * s["layer"]:2 * s["layer"] + 2, b, h, at] = _pack(new)
    status = (~torch.isfinite(new)).any(-1).any(-1).any(0).to(torch.int32)
    k, v = _read_plain(s)
    return dict(k=k, v=v, status=status)


# -- the same from the definitions, in 64 bits --------------------------------
def _values64(x):
    """What a row of numbers is held as."""
    D = x.shape[-1]
    g = x.double().unflatten(-1, (8, D // 8))
    size = g.abs().amax(-1, keepdim=True)
    last = torch.zeros_like(size)
    for e in reversed(range(D // 8)):                                 # the first of the largest decides the sign
        last = torch.where(g[..., e:e + 1].abs() == size, g[..., e:e + 1], last)
    m, e = torch.frexp(last)
    step = -torch.ldexp(torch.round(m * 32.0) / 32.0, e) / 8.0
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
    t = torch.ldexp(1.0 + m.double() / 128.0, e - 127 + 16) * torch.where(hi >= 128, -1.0, 1.0) * (e > 0)
    for x in range(D):
        word, j, odd = x // 8, (x % 8) // 2, x % 2
        byte = r[..., 4 * word + 2 * odd + j // 2]
        code = (byte >> (4 * (j % 2))) & 15
        out[..., x] = (code - 8).double() * t[..., x // (D // 8)]
    return out


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    lens, counts = _lens(c), _counts(c)
    n, H, D = c["n"], c["H"], c["D"]
    if c["op"] == "cache":
        status = torch.zeros(c["B"], n, dtype=torch.int32, device=DEV)
        return dict(k=_values64(s["k"]), v=_values64(s["v"]), status=status)
    if c["op"] == "read":
        if c["B"] * n * H * D > 1 << 26:
            return None
        got = [torch.stack([_held64(s["cache"][p, b, :, lens[b]:lens[b] + n]).transpose(0, 1) for b in range(c["B"])]) for p in (0, 1)]
        return dict(k=got[0], v=got[1])
    if work(c)["flops"] > 2e12 or c["B"] * H * c["hi"] * D > 1 << 30:
        return None
    Hq, W = c["Hq"], c["window"]
    G = Hq // H
    out = torch.zeros(c["B"], n, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.full((c["B"], n, Hq), -math.inf, dtype=torch.float64, device=DEV)
    depth, seen = _tree(c) if c["form"] == "tree" else (list(range(n)), None)
    for b in range(c["B"]):
        P, m = lens[b], counts[b]
        pos = torch.tensor([P + d for d in depth[:m]], device=DEV)
        where = torch.cat([torch.arange(P, device=DEV), pos])
        ok = torch.ones(m, P + m, dtype=torch.bool, device=DEV)
        if seen is None:
            ok = where[None, :] <= pos[:, None]
        else:
            sub = torch.zeros(m, m, dtype=torch.bool)
            for i in range(m):
                sub[i, [t for t in seen[i] if t < m]] = True
            ok[:, P:] = sub.to(DEV)
        if W:
            ok &= (pos[:, None] - where[None, :] < W) | (where[None, :] < c["sinks"])
        for h in range(H):
            K, V = _held64(s["cache"][0, b, h, :P + m]), _held64(s["cache"][1, b, h, :P + m])
            for g in range(G):
                x = (s["q"][b, :m, h * G + g].double() @ K.T) / math.sqrt(D)
                x = torch.where(ok, x, -math.inf)
                z = torch.logsumexp(x, -1)
                lse[b, :m, h * G + g] = z
                w = torch.exp(x - torch.where(torch.isfinite(z), z, torch.zeros_like(z))[:, None])
                out[b, :m, h * G + g] = w @ V
    return dict(out=out, lse=lse)
