"""Calls of the paged routed cache that a program decoding token by token makes, in plain torch and through the library.

A case is one pass of one of:
  rotary  queries and keys turned by their positions, one to three axes (time, row, column)
  append  new tokens' keys and kept value groups written to the pages of a cache
  attend  new queries over the cached tokens, optionally adding up each token's attention weight
  evict   the tokens with the most accumulated weight are chosen and moved to other pages
A cache holds pages of `page` tokens: keys K [pages, heads, page, dh]; the kept value groups of a page's tokens one after
another, V [pages, heads, slots, dh/G]; each token's group mask and first slot. A sequence is a row of page numbers and a length.
"""
import math
import random

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda"


# ---------------------------------------------------------------------------
# cases

def _rotary(name, **kw):
    return {**dict(name=name, kind="rotary", dtype="bf16", B=1, T=1, H=32, Hkv=32, dh=128, axes=3, pairs=64, pmax=4096,
                   fused=False, interleaved=False, inverse=False), **kw}


def _cache(name, kind, **kw):
    return {**dict(name=name, kind=kind, dtype="bf16", B=1, lo=0, hi=0, page=64, Hkv=32, dh=128, G=8, kv=4, kl=6), **kw}


def _append(name, **kw):
    return {**_cache(name, "append", T=1, ragged=False), **kw}


def _attend(name, **kw):
    return {**_cache(name, "attend", H=32, Tq=1, causal=False, mass=False, R=True), **kw}


def _evict(name, **kw):
    return {**_cache(name, "evict", keep=128, first=4, recent=16), **kw}


def listed():
    return [
        # one robot's next token: queries and keys of one position, latency
        _rotary("rotary-b1-token"),
        # a batch of video prefixes straight from a fused projection, three axes
        _rotary("rotary-b16-video", B=16, T=2048, Hkv=8, fused=True),
        # one new token for each of 64 sequences
        _append("append-b64-token", B=64, lo=113, hi=305, page=16, Hkv=8),
        # prefixes of up to 305 tokens written behind what is cached
        _append("append-b16-prefix", B=16, lo=0, hi=57, T=305, ragged=True),
        # the smallest attention: one robot decodes a token over its prefix and keeps the weights
        _attend("attend-b1-305", lo=305, hi=305, mass=True),
        # ordinary serving: 64 sequences of mixed lengths, four query heads a key head, fine groups
        _attend("attend-b64-gqa", B=64, lo=256, hi=2048, page=16, Hkv=8, G=16, kv=4, kl=16),
        # a chunk of 56 parallel action queries, each seeing the prefix and the actions before it
        _attend("attend-b16-actions", B=16, lo=169, hi=361, Tq=56, causal=True),
        # a long history on the full cache, weights kept for eviction: the largest
        _attend("attend-b2-131071", B=2, lo=131071, hi=131071, mass=True),
        # float32 evaluation of a smaller backbone, odd lengths
        _attend("attend-f32-dh64", dtype="f32", B=5, lo=1001, hi=3001, page=32, H=16, Hkv=4, dh=64, G=16, kv=5, kl=9),
        # one robot's cache goes back to its budget
        _evict("evict-b1-361", lo=361, hi=361, keep=176),
        # a batch of mixed lengths
        _evict("evict-b32-2048", B=32, lo=700, hi=2048, page=16, Hkv=8, G=16, kv=4, kl=16, keep=777, first=49, recent=128),
        # long histories
        _evict("evict-b4-131071", B=4, lo=90001, hi=131071, Hkv=8, keep=8192, first=64, recent=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary"] * 2 + ["append"] * 2 + ["attend"] * 5 + ["evict"] * 3)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    H, Hkv = rng.choice([(32, 32), (32, 8), (16, 16), (16, 4), (12, 4), (8, 1), (5, 5), (32, 2)])
    dh = rng.choice([128, 128, 64])
    e = 4 if dtype == "f32" else 2
    if kind == "rotary":
        B = _log(rng, 1, 64)
        return dict(kind=kind, dtype=dtype, B=B, T=max(1, min(_log(rng, 1, 4096), (32768 * 40 * 256) // (B * (H + Hkv) * dh * e))),
                    H=H, Hkv=Hkv, dh=dh, axes=rng.randint(1, 4), pairs=rng.choice([dh // 2, dh // 2, dh // 4, rng.randint(1, dh // 2)]),
                    pmax=_log(rng, 64, 1 << 20), fused=rng.random() < 0.4, interleaved=rng.random() < 0.4,
                    inverse=rng.random() < 0.3)
    G = rng.choice([4, 8, 8, 16, 32])
    c = dict(kind=kind, dtype=dtype, B=_log(rng, 1, 96), page=rng.choice([16, 32, 64, 64, 128, 256]), Hkv=Hkv, dh=dh, G=G,
             kv=rng.randint(1, G), kl=rng.randint(1, G))
    if kind == "append":
        c["T"] = max(1, min(_log(rng, 1, 700), (16 * 305 * 32 * 256) // (c["B"] * Hkv * dh * e)))
        c["lo"], c["hi"] = 0, rng.randint(0, 300)
        c["ragged"] = rng.random() < 0.5
        return c
    if kind == "evict":
        # the keys of a batch within those of the largest listed one
        c["hi"] = max(2, min(_log(rng, 40, 131071), (4 * 131071 * 8 * 256) // (c["B"] * Hkv * dh * e)))
        c["lo"] = rng.randint(1, c["hi"])
        c["keep"] = max(1, int(c["hi"] * rng.uniform(0.02, 0.15 if c["hi"] > 20000 else 0.7)))
        c["first"] = rng.randint(0, min(64, c["keep"] // 3))
        c["recent"] = rng.randint(0, c["keep"] // 3)
        return c
    c["hi"] = max(1, min(_log(rng, 1, 131071), (131071 * 32 * 256) // (c["B"] * Hkv * dh * e)))
    c["lo"] = rng.randint(0, c["hi"])
    c["H"] = H
    c["Tq"] = min(rng.choice([1, 1, 1, 1, rng.randint(2, 60)]), max(1, 10 ** 8 // (c["B"] * H * c["hi"])))
    c["causal"] = rng.random() < 0.5
    c["mass"] = rng.random() < 0.4
    c["R"] = rng.random() < 0.7
    return c


def _lens(c):
    """The lengths of a case's sequences, evenly from the longest to the shortest."""
    return [c["hi"] - (c["hi"] - c["lo"]) * i // max(1, c["B"] - 1) for i in range(c["B"])]


def _news(c):
    """New tokens of each sequence of an append: all, or evenly from all to none."""
    return [c["T"] - (c["T"] * i // c["B"] if c["ragged"] else 0) for i in range(c["B"])]


# ---------------------------------------------------------------------------
# inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _rotations(g, n, size):
    """n orthonormal size x size matrices: Walsh-Hadamard matrices between random sign flips."""
    h = torch.ones((1, 1), dtype=torch.float64, device=DEV)
    while h.shape[0] < size:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    h = h / math.sqrt(size)
    s = (torch.randint(0, 2, (3, n, size), generator=g, device=DEV) * 2 - 1).to(torch.float64)
    return torch.matmul(s[0][:, :, None] * h * s[1][:, None, :], h * s[2][:, None, :])


def _masks(c, g, *shape):
    """Group masks: a quarter of the tokens (language) keep kl groups, the others (visual) kv."""
    G = c["G"]
    r = torch.rand((*shape, G), generator=g, device=DEV).argsort(-1).argsort(-1)
    k = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.25, c["kl"], c["kv"])
    return ((r < k[..., None]).long() << torch.arange(G, device=DEV)).sum(-1).int()


def _groups(mask, G):
    """0/1 for each of a token's groups."""
    return (mask.long()[..., None] >> torch.arange(G, device=DEV)) & 1


def _pages(c, n_pages, g, dt):
    """A cache whose pages are all full."""
    P, H, dh, G = c["page"], c["Hkv"], c["dh"], c["G"]
    vcap = P * max(c["kv"], c["kl"])
    mask = _masks(c, g, n_pages, P)
    n = _groups(mask, G).sum(-1)
    return dict(K=torch.randn((n_pages, H, P, dh), generator=g, device=DEV, dtype=dt),
                V=torch.randn((n_pages, H, vcap, dh // G), generator=g, device=DEV, dtype=dt),
                mask=mask, slot=(n.cumsum(1) - n).int())


def _empty_pages(c, n_pages, dt):
    P, H, dh, G = c["page"], c["Hkv"], c["dh"], c["G"]
    return dict(K=torch.zeros((n_pages, H, P, dh), device=DEV, dtype=dt),
                V=torch.zeros((n_pages, H, P * max(c["kv"], c["kl"]), dh // G), device=DEV, dtype=dt),
                mask=torch.zeros((n_pages, P), device=DEV, dtype=torch.int32),
                slot=torch.zeros((n_pages, P), device=DEV, dtype=torch.int32))


def _table(B, width, g):
    return torch.randperm(B * width, generator=g, device=DEV).reshape(B, width).int()


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _inputs(c, seed):
    g, dt, rng = _gen(seed), DT[c["dtype"]], random.Random(seed)
    randn = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=dt)  # noqa: E731
    if c["kind"] == "rotary":
        B, T, H, Hkv, dh, n, A = (c[x] for x in ("B", "T", "H", "Hkv", "dh", "pairs", "axes"))
        if c["fused"]:
            qkv = randn(B, T, (H + 2 * Hkv) * dh)
            q = qkv[..., : H * dh].unflatten(2, (H, dh))
            k = qkv[..., H * dh: (H + Hkv) * dh].unflatten(2, (Hkv, dh))
        else:
            q, k = randn(B, T, H, dh), randn(B, T, Hkv, dh)
        i = torch.arange(n, device=DEV, dtype=torch.float64)
        axis = (i * A / n).to(torch.uint8) if not c["interleaved"] else (i % A).to(torch.uint8)
        return dict(q=q, k=k, positions=torch.randint(0, c["pmax"], (B, T, A), generator=g, device=DEV, dtype=torch.int32),
                    inv_freq=(10000.0 ** (-i / n)).float(), axis=axis)
    B, P, H, dh, G = c["B"], c["page"], c["Hkv"], c["dh"], c["G"]
    lens = _lens(c)
    rng.shuffle(lens)
    top = c["hi"] + (c["T"] if c["kind"] == "append" else 0)
    width = max(1, -(-top // P))
    s = dict(_pages(c, B * width, g, dt), table=_table(B, width, g), lens=_ints(lens))
    if c["kind"] == "append":
        new = _news(c)
        rng.shuffle(new)
        s.update(k=randn(B, c["T"], H, dh), z=randn(B, c["T"], H, dh), new_mask=_masks(c, g, B, c["T"]), n_new=_ints(new))
    elif c["kind"] == "attend":
        s["q"] = randn(B, c["Tq"], c["H"], dh)
        s["R"] = _rotations(g, H, dh).to(dt) if c["R"] else None
        if c["causal"] and c["Tq"] > 1:
            s["visible"] = (s["lens"][:, None] - torch.arange(c["Tq"] - 1, -1, -1, device=DEV, dtype=torch.int32)).clamp(min=0)
        else:
            s["visible"] = None
        s["mass"] = torch.rand((B, c["hi"]), generator=g, device=DEV) if c["mass"] else None
    else:
        # weights spread over decades, many of them equal
        m = torch.exp(2 * torch.randn((B, c["hi"]), generator=g, device=DEV))
        s["mass"] = torch.where(torch.rand((B, c["hi"]), generator=g, device=DEV) < 0.3, (m * 4).floor() / 4, m)
        s["dst_table"] = _table(B, -(-c["keep"] // P), g)
    return s


def prepare(case, seed):
    c = case
    s = dict(_inputs(c, seed), c=c)
    dt = DT[c["dtype"]]
    if c["kind"] == "attend":
        s["out"] = torch.empty_like(s["q"])
        s["mass_out"] = torch.zeros_like(s["mass"]) if c["mass"] else None
    elif c["kind"] == "evict":
        s["dst"] = _empty_pages(c, s["dst_table"].numel(), dt)
        s["mass_out"] = torch.zeros((c["B"], c["keep"]), device=DEV)
    if own:
        import paper_2608_18410_amd as rs
        if c["kind"] != "rotary":
            s["cache"] = rs.PagedCache(s["K"], s["V"], s["mask"], s["slot"])
        if c["kind"] == "attend":
            n = rs.attend_paged_workspace_size(s["cache"], c["B"], c["H"], c["Tq"], c["hi"], mass=c["mass"])
            s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
        elif c["kind"] == "evict":
            s["dst_cache"] = rs.PagedCache(**s["dst"])
            n = rs.evict_workspace_size(c["B"], c["hi"])
            s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass through the library

def _run_own(s):
    import paper_2608_18410_amd as rs
    c = s["c"]
    if c["kind"] == "rotary":
        q, k = rs.rotary(s["q"], s["k"], s["positions"], s["inv_freq"], s["axis"], interleaved=c["interleaved"],
                         inverse=c["inverse"])
        return {"q": q, "k": k}
    if c["kind"] == "append":
        rs.cache_append(s["cache"], s["k"], s["z"], s["new_mask"], s["table"], s["lens"], n_new=s["n_new"])
        return {x: s[x] for x in ("K", "V", "mask", "slot")}
    if c["kind"] == "attend":
        out = rs.attend_paged(s["q"], s["cache"], s["table"], s["lens"], s["R"], visible=s["visible"], max_len=c["hi"],
                              mass=s["mass"], decay=0.75, mass_out=s["mass_out"], workspace=s["ws"], out=s["out"])
        return {"out": out, "mass": s["mass_out"]} if c["mass"] else {"out": out}
    idx, n = rs.evict_tokens(s["mass"], s["lens"], c["keep"], first=c["first"], recent=c["recent"], workspace=s["ws"])
    rs.cache_compact(s["cache"], s["table"], idx, n, s["dst_cache"], s["dst_table"], mass=s["mass"], mass_out=s["mass_out"])
    return {"idx": idx, "n": n, "mass_out": s["mass_out"], **s["dst"]}


# ---------------------------------------------------------------------------
# the same in plain torch

def _turn(x, cos, sin, n, interleaved):
    """Pairs (i, i + n), or (2i, 2i + 1), of the last dimension turned; the dimensions past 2n stay."""
    x = x.float()
    a, b = (x[..., 0: 2 * n: 2], x[..., 1: 2 * n: 2]) if interleaved else (x[..., :n], x[..., n: 2 * n])
    ya, yb = a * cos - b * sin, a * sin + b * cos
    y = torch.stack((ya, yb), -1).flatten(-2) if interleaved else torch.cat((ya, yb), -1)
    return torch.cat((y, x[..., 2 * n:]), -1)


def _plain_rotary(s):
    c = s["c"]
    a = s["positions"].double()[..., s["axis"].long()] * s["inv_freq"].double()
    cos, sin = torch.cos(a).float()[:, :, None], torch.sin(a).float()[:, :, None]
    sin = -sin if c["inverse"] else sin
    return {x: _turn(s[x], cos, sin, c["pairs"], c["interleaved"]).to(s[x].dtype) for x in ("q", "k")}


def _put(dst, page, row, take, k, z_groups, mask, page_start):
    """Tokens [B, T] into pages: keys k [B, T, H, dh], groups z [B, T, H, G, ds]; `take` says which are there, page_start
    the slots taken before a token's page-mates among them."""
    G = z_groups.shape[3]
    bits = _groups(mask, G) * take[..., None]
    n = bits.sum(-1)
    before = n.cumsum(1) - n
    first = torch.cat((torch.ones_like(page[:, :1], dtype=torch.bool), page[:, 1:] != page[:, :-1]), 1)
    base = torch.where(first, before, torch.zeros_like(before)).cummax(1).values
    start = before - base + page_start
    p, r = page[take], row[take]
    dst["K"][p, :, r] = k[take]
    dst["mask"][p, r] = mask[take]
    dst["slot"][p, r] = start[take].int()
    at = start[..., None] + bits.cumsum(-1) - bits
    kept = bits > 0
    dst["V"][page[..., None].expand_as(kept)[kept], :, at[kept]] = z_groups.transpose(2, 3)[kept]


def _plain_append(s):
    c = s["c"]
    P, G = c["page"], c["G"]
    lens = s["lens"].long()[:, None]
    j = torch.arange(c["T"], device=DEV)[None]
    t = lens + j
    page, row = torch.gather(s["table"].long(), 1, t // P), t % P
    take = j < s["n_new"].long()[:, None]
    # the slots that the cached tokens of the first page have taken
    prev = (lens - 1).clamp(min=0)
    pp, pr = torch.gather(s["table"].long(), 1, prev // P), prev % P
    used = s["slot"][pp, pr].long() + _groups(s["mask"][pp, pr], G).sum(-1)
    used = torch.where((lens % P > 0) & (t // P == lens // P), used, torch.zeros_like(used))
    _put(s, page, row, take, s["k"], s["z"].unflatten(3, (G, -1)), s["new_mask"], used)
    return {x: s[x] for x in ("K", "V", "mask", "slot")}


def _fetch(s, page, row):
    """Keys [.., Hkv, dh], groups [.., Hkv, G, ds] (dropped ones zero) and masks of cached tokens."""
    G = s["c"]["G"]
    m = s["mask"][page, row]
    bits = _groups(m, G)
    at = (s["slot"][page, row].long()[..., None] + bits.cumsum(-1) - bits).clamp(max=s["V"].shape[2] - 1)
    z = s["V"][page[..., None], :, at] * bits[..., None, None].to(s["V"].dtype)
    return s["K"][page, :, row], z.transpose(-3, -2), m


def _plain_attend(s):
    c = s["c"]
    P, H, Hkv, dh, Tq, L = c["page"], c["H"], c["Hkv"], c["dh"], c["Tq"], c["hi"]
    t = torch.arange(L, device=DEV)
    step = max(1, (1 << 30) // max(1, L * Hkv * dh * 4))  # sequences at a time: about 1 GiB of keys
    for b in range(0, c["B"], step):
        sl = slice(b, b + step)
        K, z, _ = _fetch(s, s["table"][sl].long()[:, t // P], (t % P).expand(s["table"][sl].shape[0], L))
        K, z = K.float().transpose(1, 2), z.float().flatten(3).transpose(1, 2)  # [b, Hkv, L, dh]
        q = s["q"][sl].float().unflatten(2, (Hkv, H // Hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [b, Hkv, rep * Tq, dh]
        x = torch.matmul(q, K.transpose(2, 3)) / math.sqrt(dh)
        see = s["lens"][sl].long()[:, None].expand(-1, Tq)
        if s["visible"] is not None:
            see = torch.minimum(see, s["visible"][sl].long())
        see = (t < see[..., None]).repeat(1, H // Hkv, 1)[:, None]
        top = torch.where(see, x, -1e30).amax(-1, keepdim=True)
        e = torch.where(see, torch.exp(x - top), 0.0)
        p = e / e.sum(-1, keepdim=True).clamp(min=1e-30)
        u = torch.matmul(p, z)
        if s["R"] is not None:
            u = torch.matmul(u, s["R"].float().transpose(1, 2))
        s["out"][sl] = u.unflatten(2, (H // Hkv, Tq)).permute(0, 3, 1, 2, 4).flatten(2, 3).to(s["out"].dtype)
        if c["mass"]:
            m = 0.75 * s["mass"][sl] + p.sum((1, 2))
            s["mass_out"][sl] = torch.where(t < s["lens"][sl][:, None], m, s["mass_out"][sl])
    return {"out": s["out"], "mass": s["mass_out"]} if c["mass"] else {"out": s["out"]}


def _plain_evict(s):
    c = s["c"]
    P, keep, L = c["page"], c["keep"], c["hi"]
    lens = s["lens"].long()[:, None]
    t = torch.arange(L, device=DEV)[None]
    key = torch.where((t < c["first"]) | (t >= lens - c["recent"]), math.inf, s["mass"])
    key = torch.where(t < lens, key, -math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :keep]
    n = lens.clamp(max=keep)
    j = torch.arange(keep, device=DEV)[None]
    if order.shape[1] < keep:
        order = torch.cat((order, order.new_full((order.shape[0], keep - order.shape[1]), L)), 1)
    idx = torch.where(j < n, order, L).sort(1).values
    take = j < n
    at = torch.where(take, idx, 0)
    k, z, m = _fetch(s, torch.gather(s["table"].long(), 1, at // P), at % P)
    page = torch.repeat_interleave(s["dst_table"].long(), P, 1)[:, :keep]
    _put(s["dst"], page, (j % P).expand_as(page), take, k, z, m, 0)
    s["mass_out"][take] = torch.gather(s["mass"], 1, at)[take]
    return {"idx": torch.where(take, idx, -1).int(), "n": n[:, 0].int(), "mass_out": s["mass_out"], **s["dst"]}


def run(state):
    if own:
        return _run_own(state)
    return {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend,
            "evict": _plain_evict}[state["c"]["kind"]](state)


# ---------------------------------------------------------------------------
# the least work of a pass

def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rotary":
        n = c["B"] * c["T"]
        return {"bytes": n * (2 * (c["H"] + c["Hkv"]) * c["dh"] * e + 4 * c["axes"]) + 5 * c["pairs"],
                "flops": n * ((c["H"] + c["Hkv"]) * c["pairs"] * 6 + 40 * c["pairs"])}
    row = c["Hkv"] * c["dh"] * e
    groups = (0.25 * c["kl"] + 0.75 * c["kv"]) / c["G"]  # kept share of a value
    if c["kind"] == "append":
        n = sum(_news(c))
        return {"bytes": int(n * (2 * row * (1 + groups) + 16)), "flops": 0}
    if c["kind"] == "evict":
        n = sum(min(x, c["keep"]) for x in _lens(c))
        return {"bytes": int(4 * sum(_lens(c)) + n * (2 * row * (1 + groups) + 28)), "flops": 0}
    tokens, seen = sum(_lens(c)), 0
    for x in _lens(c):
        seen += sum(max(0, x - i) for i in range(c["Tq"])) if c["causal"] else x * c["Tq"]
    heads = c["B"] * c["Tq"] * c["H"] * c["dh"]
    by = tokens * (row * (1 + groups) + 8 + (8 if c["mass"] else 0)) + 2 * heads * e
    fl = 2 * seen * c["H"] * c["dh"] * (1 + groups)
    if c["R"]:
        by += c["Hkv"] * c["dh"] ** 2 * e
        fl += 2 * heads * c["dh"]
    return {"bytes": int(by), "flops": int(fl)}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the formulas, one sequence at a time

def _dense(s, b, n, c):
    """Keys and masked values [n, Hkv, dh] of sequence b's first n tokens, from its pages."""
    P, G = c["page"], c["G"]
    ks, vs = [], []
    for i, p in enumerate(s["table"][b].tolist()[: -(-n // P)]):
        m = min(P, n - i * P)
        ks.append(s["K"][p, :, :m].double().transpose(0, 1))
        on = _groups(s["mask"][p, :m], G).bool()  # [m, G]
        v = torch.zeros((m, G, c["Hkv"], c["dh"] // G), dtype=torch.float64, device=DEV)
        tok, grp = on.nonzero(as_tuple=True)  # a page's groups lie in this order
        v[tok, grp] = s["V"][p, :, : tok.numel()].double().transpose(0, 1)
        vs.append(v.transpose(1, 2).flatten(2))
    return torch.cat(ks), torch.cat(vs)


def _exact_rotary(s, c):
    n, o = c["pairs"], {}
    ang = torch.stack([s["positions"][..., int(a)].double() * f.double() for a, f in zip(s["axis"].tolist(), s["inv_freq"])], -1)
    w = torch.polar(torch.ones_like(ang), -ang if c["inverse"] else ang)[:, :, None]
    for x in ("q", "k"):
        y = s[x].double().clone()
        i = torch.arange(n, device=DEV)
        i, j = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + n)
        zc = torch.complex(y[..., i], y[..., j]) * w
        y[..., i], y[..., j] = zc.real, zc.imag
        o[x] = y
    return o


def _exact_append(s, c):
    P, G = c["page"], c["G"]
    K, V = s["K"].double(), s["V"].double()
    on = _groups(s["new_mask"], G).bool().cpu()
    table, lens, new = s["table"].tolist(), s["lens"].tolist(), s["n_new"].tolist()
    old = _groups(s["mask"], G).sum(-1).cpu()
    for b in range(c["B"]):
        used = int(old[table[b][lens[b] // P], : lens[b] % P].sum()) if lens[b] % P else 0
        for j in range(new[b]):
            p, r = table[b][(lens[b] + j) // P], (lens[b] + j) % P
            used = 0 if r == 0 else used
            g = on[b, j].nonzero()[:, 0]
            K[p, :, r] = s["k"][b, j].double()
            V[p, :, used: used + len(g)] = s["z"][b, j].double().unflatten(1, (G, -1))[:, g.to(DEV)]
            used += len(g)
    return {"K": K, "V": V, "mask": None, "slot": None}


def _exact_attend(s, c):
    H, Hkv, dh, Tq = c["H"], c["Hkv"], c["dh"], c["Tq"]
    out = torch.zeros((c["B"], Tq, H, dh), dtype=torch.float64, device=DEV)
    mass = torch.zeros((c["B"], c["hi"]), dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        see = [n] * Tq if s["visible"] is None else [min(n, x) for x in s["visible"][b].tolist()]
        K, V = _dense(s, b, n, c)
        hidden = torch.arange(n, device=DEV)[None] >= torch.tensor(see, device=DEV)[:, None]  # [Tq, n]
        for h in range(H):
            kv = h // (H // Hkv)
            x = (s["q"][b, :, h].double() @ K[:, kv].T) * dh ** -0.5
            p = torch.softmax(x.masked_fill(hidden, -math.inf), -1).nan_to_num(0.0)
            u = p @ V[:, kv]
            out[b, :, h] = u if s["R"] is None else u @ s["R"][kv].double().T
            mass[b, :n] += p.sum(0)
        if c["mass"]:
            mass[b, :n] += 0.75 * s["mass"][b, :n].double()
    return {"out": out, "mass": mass} if c["mass"] else {"out": out}


def _exact_evict(s, c):
    P, G, keep = c["page"], c["G"], c["keep"]
    dst = _empty_pages(c, s["dst_table"].numel(), DT[c["dtype"]])
    K, V, mass = dst["K"].double(), dst["V"].double(), torch.zeros((c["B"], keep), dtype=torch.float64, device=DEV)
    table = s["dst_table"].tolist()
    for b, n in enumerate(s["lens"].tolist()):
        t = torch.arange(n, device=DEV)
        if n > keep:
            safe = (t < c["first"]) | (t >= n - c["recent"])
            free = t[~safe]
            best = free[torch.argsort(-s["mass"][b, free].double(), stable=True)[: keep - c["first"] - c["recent"]]]
            t = torch.cat((t[safe], best)).sort().values
        sp = s["table"][b].long()[t // P]
        mass[b, : len(t)] = s["mass"][b, t].double()
        on = _groups(s["mask"][sp, t % P], G).bool()
        old = s["slot"][sp, t % P].long()
        for i in range(0, len(t), P):
            p, e = table[b][i // P], slice(i, i + P)
            K[p, :, : len(t[e])] = s["K"][sp[e], :, t[e] % P].double().transpose(0, 1)
            cnt = on[e].sum(1)
            tok = torch.repeat_interleave(torch.arange(len(t[e]), device=DEV), cnt)
            nth = torch.arange(len(tok), device=DEV) - torch.repeat_interleave(cnt.cumsum(0) - cnt, cnt)
            V[p, :, : len(tok)] = s["V"][sp[e][tok], :, old[e][tok] + nth].double().transpose(0, 1)
    return {"idx": None, "n": None, "mass_out": mass, "K": K, "V": V, "mask": None, "slot": None}


def exact(case, seed):
    s = _inputs(case, seed)
    return {"rotary": _exact_rotary, "append": _exact_append, "attend": _exact_attend,
            "evict": _exact_evict}[case["kind"]](s, case)
