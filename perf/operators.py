"""Timed cases of the paged key/value cache: one serving step's page and slot maps, the queries'
and keys' norm and rotation with the cache write, and the attention that reads the cache.

A step of a serving loop over several requests (robots, cameras, dialogues) first gives every
new token a place in the cache (`paged_slots`), then in every layer normalises and rotates the
projected queries and keys and writes keys and values to their places (`qk_norm_rope`), and lets
the new tokens attend to their request's whole history through its block table
(`paged_attention`).

`listed()` gives the named cases, `draw(rng)` another one of the same ranges, `prepare(case,
seed)` what a program holds before the call, `run(state)` one pass (`own`: through the library,
else in elementary torch operations in 32 bits), `work(case)` the bytes and operations it cannot
do without, `exact(case, seed)` the outputs in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6
BASE = 10000.0
WORKSPACE_BYTES = 64 << 20  # of the attention's key splits


# ----------------------------------------------------------------------------- the cases

def listed():
    return [
        # one robot's action chunk joins its 816-token prefix (3 x 256 image + 48 text tokens)
        {"name": "slots_chunk", "op": "slots", "reqs": 1, "c_lo": 816, "c_hi": 816, "q_lo": 50, "q_hi": 50,
         "page": 16, "lens": 1},
        # a decode step of a large fleet: one token each, some requests idle
        {"name": "slots_decode_r1000", "op": "slots", "reqs": 1000, "c_lo": 0, "c_hi": 4000, "q_lo": 0, "q_hi": 1,
         "page": 16, "lens": 2},
        # many prompts admitted at once, ragged lengths
        {"name": "slots_prompts_r512", "op": "slots", "reqs": 512, "c_lo": 0, "c_hi": 300, "q_lo": 1, "q_hi": 1632,
         "page": 64, "lens": 3},
        # one decoded action token: 8 query heads on one key/value head, a layer's latency
        {"name": "qk_decode_t1", "op": "qk", "tokens": 1, "H": 8, "Hk": 1, "d": 128, "axes": 1, "norm": True,
         "packed": False, "page": 16},
        # image and text tokens of a prefix (three position axes) from one packed projection
        {"name": "qk_prefix_t816_axes3", "op": "qk", "tokens": 816, "H": 32, "Hk": 8, "d": 128, "axes": 3,
         "norm": True, "packed": True, "page": 16},
        # a prefill batch of a 2B backbone: heads of 256, rotation and cache write without a norm
        {"name": "qk_prefill_t16000_d256", "op": "qk", "tokens": 16000, "H": 8, "Hk": 1, "d": 256, "axes": 1,
         "norm": False, "packed": False, "page": 64},
        # one decoded token over one robot's prefix and chunk: latency
        {"name": "attn_decode_r1", "op": "attn", "reqs": 1, "c_lo": 866, "c_hi": 866, "q_lo": 1, "q_hi": 1, "H": 8,
         "Hk": 1, "d": 128, "page": 16, "mask": "causal", "prefix": 0, "cap": 0.0, "window": 0, "lens": 4},
        # the action expert's 50-token chunk, all of it and the whole prefix visible
        {"name": "attn_chunk_m50", "op": "attn", "reqs": 1, "c_lo": 816, "c_hi": 816, "q_lo": 50, "q_hi": 50, "H": 8,
         "Hk": 1, "d": 128, "page": 16, "mask": "full", "prefix": 0, "cap": 0.0, "window": 0, "lens": 5},
        # a decode batch with ragged long histories: the cache's bandwidth
        {"name": "attn_decode_r64_16k", "op": "attn", "reqs": 64, "c_lo": 100, "c_hi": 16383, "q_lo": 1, "q_hi": 1,
         "H": 32, "Hk": 8, "d": 128, "page": 64, "mask": "causal", "prefix": 0, "cap": 0.0, "window": 0, "lens": 6},
        # drafted tokens checked in a batch: a few queries each, heads of 64, scores capped, sliding window
        {"name": "attn_drafts_r24_d64", "op": "attn", "reqs": 24, "c_lo": 0, "c_hi": 3000, "q_lo": 1, "q_hi": 7,
         "H": 14, "Hk": 2, "d": 64, "page": 32, "mask": "causal", "prefix": 0, "cap": 50.0, "window": 1024, "lens": 7},
        # a 2B backbone's prefill: heads of 256, the 768 image tokens visible to one another, the text causal
        {"name": "attn_prefix_m816_d256", "op": "attn", "reqs": 2, "c_lo": 0, "c_hi": 0, "q_lo": 816, "q_hi": 816,
         "H": 8, "Hk": 1, "d": 256, "page": 16, "mask": "prefix", "prefix": 768, "cap": 0.0, "window": 0, "lens": 8},
        # a chunk of a long prompt over what is cached already: the tensor cores' rate
        {"name": "attn_chunk_4096_of_16384", "op": "attn", "reqs": 1, "c_lo": 12288, "c_hi": 12288, "q_lo": 4096,
         "q_hi": 4096, "H": 32, "Hk": 8, "d": 128, "page": 64, "mask": "causal", "prefix": 0, "cap": 0.0,
         "window": 0, "lens": 9},
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _draw_once(rng):
    op = rng.choice(["slots", "qk", "attn", "attn", "attn"])
    if op == "slots":
        reqs = _log(rng, 1, 1000)
        q_hi = rng.choice([1, _log(rng, 2, max(2, min(1632, 400000 // reqs)))])
        return {"op": op, "reqs": reqs, "c_lo": 0, "c_hi": _log(rng, 1, 8000), "q_lo": rng.choice([0, 1]), "q_hi": q_hi,
                "page": rng.choice([16, 32, 64, 128]), "lens": rng.randrange(1 << 30)}
    d = rng.choice([64, 128, 128, 256])
    Hk = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 7, 8])
    page = rng.choice([16, 32, 64, 128])
    if op == "qk":
        return {"op": op, "tokens": _log(rng, 1, 16000), "H": Hk * G, "Hk": Hk, "d": d, "axes": rng.choice([1, 3]),
                "norm": rng.random() < 0.6, "packed": rng.random() < 0.5, "page": page}
    kind = rng.choice(["decode", "drafts", "prefill"])
    reqs = rng.choice([1, _log(rng, 1, 64)])
    c_hi = _log(rng, 16, 16000)
    q_hi = 1 if kind == "decode" else _log(rng, 2, 16) if kind == "drafts" else _log(rng, 16, 4096)
    return {"op": op, "reqs": reqs, "c_lo": rng.choice([0, c_hi // 2]), "c_hi": c_hi,
            "q_lo": rng.choice([0, q_hi]) if reqs > 1 else q_hi, "q_hi": q_hi, "H": Hk * G, "Hk": Hk, "d": d,
            "page": page, "mask": rng.choice(["causal", "causal", "prefix", "full"]), "prefix": _log(rng, 1, 1000),
            "cap": rng.choice([0.0, 0.0, 30.0, 50.0]), "window": rng.choice([0, 0, 0, _log(rng, 1, 4096)]),
            "lens": rng.randrange(1 << 30)}


def _cost(case):
    """Seconds at the card's rates, and GB that the plain form's padded tensors take."""
    w = work(case)
    gb = 0.0
    if case["op"] == "attn":
        q, kv = _lengths(case)
        gb = 4e-9 * len(q) * max(kv) * (max(q) * case["H"] + 2 * case["Hk"] * case["d"])
    return w["bytes"] / 6.8e12 + w["flops"] / 1.9e15, gb


def draw(rng):
    """Another case of the listed ranges: sizes over their logarithm from one token to the largest
    listed ones, no costlier than the largest."""
    largest = [_cost(c) for c in listed()]
    most = [max(x[i] for x in largest) for i in (0, 1)]
    while True:
        case = _draw_once(rng)
        cost = _cost(case)
        if all(c <= m for c, m in zip(cost, most)):
            return case


def _lengths(case):
    """New and total tokens of every request."""
    r = random.Random(case["lens"])
    cached = [r.randint(case["c_lo"], case["c_hi"]) for _ in range(case["reqs"])]
    new = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["reqs"])]
    if sum(new) == 0:
        new[0] = 1
    return new, [c + n for c, n in zip(cached, new)]


def _range(case, p, kv, prefix):
    """Keys [lo, hi) that the query at position p sees."""
    return (max(0, p - case["window"] + 1) if case["window"] else 0), min(kv, max(p + 1, prefix))


def _prefix_of(case, kv):
    return {"causal": 0, "prefix": min(case["prefix"], kv), "full": kv}[case["mask"]]


# ----------------------------------------------------------------------------- inputs

def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _pages(case, kv, g, spare):
    """Pages in a random order of the cache: the block table (-1 past a request's pages) and what is left."""
    page = case["page"]
    need = [-(-n // page) for n in kv]
    n_pages = sum(need) + spare
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    width = max(1, max(need))
    need_t = _ints(need, torch.int64)
    first = need_t.cumsum(0) - need_t
    col = torch.arange(width, device="cuda")[None]
    table = torch.where(col < need_t[:, None], perm[(first[:, None] + col).clamp(max=n_pages - 1)], -1).to(torch.int32)
    return table, perm[sum(need):].contiguous(), n_pages


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = {"device": "cuda"}

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, **dev) * scale).to(torch.bfloat16)

    s = {"case": case}
    if case["op"] == "slots":
        new, kv = _lengths(case)
        cached = [a - b for a, b in zip(kv, new)]
        page = case["page"]
        want = sum(-(-n // page) for n in kv) - sum(-(-n // page) for n in cached)
        table, free, _ = _pages(case, cached, g, want + 40)
        width = max(-(-n // page) for n in kv)
        s["table"] = torch.full((len(kv), width + 4), -1, dtype=torch.int32, **dev)
        s["table"][:, :min(width, table.shape[1])] = table[:, :width]
        T = sum(new)
        s |= {"cached": _ints(cached), "added": _ints(new), "free": free, "used": _ints([17]), "page": page,
              "q_start": torch.empty(len(kv) + 1, dtype=torch.int32, **dev),
              "kv_len": torch.empty(len(kv), dtype=torch.int32, **dev),
              "slots": torch.empty(T, dtype=torch.int64, **dev),
              "positions": torch.empty(T, dtype=torch.int32, **dev),
              "used_out": torch.empty(1, dtype=torch.int32, **dev)}
        return s
    H, Hk, d, page = case["H"], case["Hk"], case["d"], case["page"]
    if case["op"] == "qk":
        T, axes, half = case["tokens"], case["axes"], d // 2
        # the projections' outputs: one packed matrix or three
        if case["packed"]:
            packed = normal(T, (H + 2 * Hk) * d)
            s["q"], s["k"], s["v"] = packed.split([H * d, Hk * d, Hk * d], dim=1)
        else:
            s["q"], s["k"], s["v"] = normal(T, H * d), normal(T, Hk * d), normal(T, Hk * d)
        gamma = 1.0 + 0.1 * torch.randn(2, d, generator=g, **dev)
        s["q_gamma"], s["k_gamma"] = (gamma[0], gamma[1]) if case["norm"] else (None, None)
        if axes == 1:
            s["positions"] = (torch.arange(T, **dev) + seed % 1000).to(torch.int32)[None]
        else:  # three images of a 16 x 16 grid, then text: time, height, width
            t = torch.arange(T, **dev)
            img, at = t // 256, t % 256
            text = t >= 768
            s["positions"] = torch.stack([torch.where(text, t - 704, img), torch.where(text, t - 704, img + at // 16),
                                          torch.where(text, t - 704, img + at % 16)]).to(torch.int32).contiguous()
        # pairs of a head by axis: a quarter turns with time, the rest with height and width
        parts = [half] if axes == 1 else [half // 4, half * 3 // 8, half - half // 4 - half * 3 // 8]
        s["axis_of_pair"] = [a for a, n in enumerate(parts) for _ in range(n)]
        s["axis_index"] = _ints(s["axis_of_pair"], torch.int64)
        n_pages = -(-T // page) + 3
        order = torch.randperm(n_pages, generator=g, **dev)
        t = torch.arange(T, **dev)
        s["slots"] = order[t // page] * page + t % page
        s["k_cache"], s["v_cache"] = normal(n_pages, page, Hk, d), normal(n_pages, page, Hk, d)
        s["q_out"] = torch.empty(T, H * d, dtype=torch.bfloat16, **dev)
        return s
    new, kv = _lengths(case)
    s["table"], _, n_pages = _pages(case, kv, g, 2)
    s["q"] = normal(sum(new), H * d)
    s["k_cache"], s["v_cache"] = normal(n_pages, page, Hk, d), normal(n_pages, page, Hk, d)
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    s["q_start"], s["kv_len"], s["max_q"] = _ints(start), _ints(kv), max(new)
    s["prefix"] = None if case["mask"] == "causal" else _ints([_prefix_of(case, n) for n in kv])
    s["scale"] = d ** -0.5
    s["o"] = torch.empty(sum(new), H * d, dtype=torch.bfloat16, **dev)
    s["workspace"] = torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, **dev)
    return s


# ----------------------------------------------------------------------------- one pass

def run(state):
    if own:
        return {"slots": _own_slots, "qk": _own_qk, "attn": _own_attn}[state["case"]["op"]](state)
    return {"slots": _plain_slots, "qk": _plain_qk, "attn": _plain_attn}[state["case"]["op"]](state)


def _own_slots(s):
    import paper_2607_02501_gb300 as emb
    emb.emb_paged_slots(s["cached"], s["added"], s["free"], s["used"], s["table"], s["q_start"], s["kv_len"], s["slots"],
                        s["positions"], s["used_out"], s["page"])
    return {k: s[k] for k in ("table", "q_start", "kv_len", "slots", "positions", "used_out")}


def _own_qk(s):
    import paper_2607_02501_gb300 as emb
    emb.emb_qk_norm_rope(s["q"], s["k"], s["v"], s["q_out"], s["k_cache"], s["v_cache"], s["slots"], s["positions"],
                         q_gamma=s["q_gamma"], k_gamma=s["k_gamma"], eps=EPS, axis_of_pair=s["axis_of_pair"], base=BASE)
    return {k: s[k] for k in ("q_out", "k_cache", "v_cache")}


def _own_attn(s):
    import paper_2607_02501_gb300 as emb
    c = s["case"]
    emb.emb_paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["q_start"], s["kv_len"], s["o"],
                            s["scale"], s["max_q"], s["workspace"], prefix=s["prefix"], cap=c["cap"], window=c["window"])
    return s["o"]


def _plain_slots(s):
    page, table, T = s["page"], s["table"], s["slots"].shape[0]
    R, width = table.shape
    cached, added = s["cached"].long(), s["added"].long()
    kv = cached + added
    q_end = added.cumsum(0)
    q_start = torch.cat([q_end.new_zeros(1), q_end])
    # requests take their new pages from the free list one after another
    have, want = (cached + page - 1) // page, (kv + page - 1) // page
    need = want - have
    first = s["used"].long() + need.cumsum(0) - need
    col = torch.arange(width, device="cuda")[None]
    at = first[:, None] + col - have[:, None]
    n_free = s["free"].shape[0]
    taken = torch.where(at < n_free, s["free"][at.clamp(0, n_free - 1)], -1)
    table = torch.where((col >= have[:, None]) & (col < want[:, None]), taken, table)
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(q_end, t, right=True)
    pos = cached[r] + t - q_start[r]
    pages = table[r, pos // page].long()
    slots = torch.where(pages >= 0, pages * page + pos % page, -1)
    return {"table": table, "q_start": q_start.int(), "kv_len": kv.int(), "slots": slots, "positions": pos.int(),
            "used_out": (s["used"] + need.sum()).int()}


def _plain_qk(s):
    c = s["case"]
    T, H, Hk, d = c["tokens"], c["H"], c["Hk"], c["d"]
    half = d // 2
    freq = BASE ** (torch.arange(half, device="cuda") * (-2.0 / d))
    angle = s["positions"][s["axis_index"]].T.float() * freq
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def rotated(x, heads, gamma):
        x = x.reshape(T, heads, d).float()
        if gamma is not None:
            x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * gamma
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)

    s["q_out"].copy_(rotated(s["q"], H, s["q_gamma"]).view(T, H * d))
    s["k_cache"].view(-1, Hk, d)[s["slots"]] = rotated(s["k"], Hk, s["k_gamma"])
    s["v_cache"].view(-1, Hk, d)[s["slots"]] = s["v"].reshape(T, Hk, d)
    return {k: s[k] for k in ("q_out", "k_cache", "v_cache")}


def _plain_attn(s):
    c = s["case"]
    H, Hk, d, page, G = c["H"], c["Hk"], c["d"], c["page"], c["H"] // c["Hk"]
    table, mq, T = s["table"], s["max_q"], s["q"].shape[0]
    R, L = table.shape[0], table.shape[1] * page
    start, kv = s["q_start"].long(), s["kv_len"].long()
    n_new = start[1:] - start[:-1]
    i = torch.arange(mq, device="cuda")
    # queries padded to the longest request's, keys gathered through the block tables
    q = s["q"].view(T, Hk, G, d)[(start[:-1, None] + i).clamp(max=T - 1)]                 # [R][mq][Hk][G][d]
    q = q.permute(0, 2, 3, 1, 4).reshape(R, Hk, G * mq, d).float()
    pages = table.clamp(min=0).long()
    k = s["k_cache"][pages].view(R, L, Hk, d).permute(0, 2, 3, 1).float()                  # [R][Hk][d][L]
    x = (q @ k).view(R, Hk, G, mq, L) * s["scale"]
    del q, k
    if c["cap"]:
        x = torch.tanh(x / c["cap"]) * c["cap"]
    p = (kv - n_new)[:, None] + i                                                         # positions [R][mq]
    j = torch.arange(L, device="cuda")
    hi = p + 1 if s["prefix"] is None else torch.maximum(p + 1, s["prefix"].long()[:, None])
    seen = (j < hi[..., None]) & (j < kv[:, None, None])
    if c["window"]:
        seen &= j > p[..., None] - c["window"]
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v = s["v_cache"][pages].view(R, L, Hk, d).permute(0, 2, 1, 3).float()
    v = v.masked_fill_((j >= kv[:, None])[:, None, :, None], 0.0)                          # past a request's end: anything
    o = (x.view(R, Hk, G * mq, L) @ v).view(R, Hk, G, mq, d) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(R, mq, H * d).to(torch.bfloat16)
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(start[1:], t, right=True)
    return o[r, t - start[r]]


# ----------------------------------------------------------------------------- what a pass needs

def work(case):
    if case["op"] == "slots":
        new, kv = _lengths(case)
        page = case["page"]
        partial = sum((n - a) % page != 0 for n, a in zip(kv, new))  # a begun page is looked up
        taken = sum(-(-n // page) - -(-(n - a) // page) for n, a in zip(kv, new))
        return {"bytes": 12 * sum(new) + 16 * len(kv) + 8 * taken + 4 * partial, "flops": 0}
    H, Hk, d = case["H"], case["Hk"], case["d"]
    if case["op"] == "qk":
        T = case["tokens"]
        return {"bytes": T * (2 * (H + 2 * Hk) * d * 2 + 8 + 4 * case["axes"]), "flops": T * (H + Hk) * d * (6 if case["norm"] else 3)}
    new, kv = _lengths(case)
    keys = pairs = 0
    for n, total in zip(new, kv):
        if n == 0:
            continue
        f = _prefix_of(case, total)
        spans = [_range(case, total - n + i, total, f) for i in range(n)]
        pairs += sum(max(0, hi - lo) for lo, hi in spans)
        keys += max(hi for _, hi in spans) - min(lo for lo, _ in spans)
    return {"bytes": 2 * sum(new) * H * d * 2 + 2 * keys * Hk * d * 2 + 4 * keys // case["page"] + 8 * len(kv),
            "flops": 4 * pairs * H * d}


# ----------------------------------------------------------------------------- 64-bit outputs

def exact(case, seed):
    """The outputs in 64 bits, request by request and head by head."""
    s = prepare(case, seed)
    if case["op"] == "slots":
        return None  # whole numbers
    H, Hk, d, page = case["H"], case["Hk"], case["d"], case["page"]
    if case["op"] == "qk":
        T, half = case["tokens"], d // 2
        turn = torch.zeros(T, half, dtype=torch.float64, device="cuda")
        for i in range(half):
            turn[:, i] = s["positions"][s["axis_of_pair"][i]].double() * math.pow(BASE, -2.0 * i / d)
        spin = torch.polar(torch.ones_like(turn), turn)
        outs = {}
        for name, heads, gamma in (("q", H, s["q_gamma"]), ("k", Hk, s["k_gamma"])):
            x = s[name].reshape(T, heads, d).double()
            if gamma is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS) * gamma.double()
            z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * spin[:, None]
            outs[name] = torch.cat([z.real, z.imag], -1)
        caches = {}
        for name, rows in (("k_cache", outs["k"]), ("v_cache", s["v"].reshape(T, Hk, d).double())):
            c = s[name].double()
            c[s["slots"] // page, s["slots"] % page] = rows
            caches[name] = c
        return {"q_out": outs["q"].reshape(T, H * d), **caches}
    new, kv = _lengths(case)
    G = H // Hk
    out = torch.zeros(sum(new), H, d, dtype=torch.float64, device="cuda")
    at = 0
    for r, (n, total) in enumerate(zip(new, kv)):
        if n == 0:
            continue
        f = _prefix_of(case, total)
        idx = torch.arange(total, device="cuda")
        page_of = s["table"][r][idx // page].long()
        spans = torch.tensor([_range(case, total - n + i, total, f) for i in range(n)], device="cuda")
        seen = (idx >= spans[:, :1]) & (idx < spans[:, 1:])
        for g in range(Hk):
            k = s["k_cache"][page_of, idx % page, g].double()
            v = s["v_cache"][page_of, idx % page, g].double()
            for h in range(g * G, (g + 1) * G):
                z = s["q"][at:at + n, h * d:(h + 1) * d].double() @ k.T * s["scale"]
                if case["cap"]:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                z = torch.where(seen, z, -math.inf)
                w = torch.exp(z - z.amax(1, keepdim=True))
                out[at:at + n, h] = w @ v / w.sum(1, keepdim=True)
        at += n
    return out.reshape(sum(new), H * d)
