"""Timed cases of the paged key/value cache in 8 bits: queries and keys normalised, rotated and keys and values stored,
stored rows read back, and the attention that reads the cache.

The cache holds e4m3 codes with one power of two for each block of 16 places of a page and head. `store` appends a
step's tokens (a block that is gone on with is re-encoded where the new tokens need a larger power), `read` expands rows
to bf16, `attention` lets new tokens attend to their request's history through its block table.

`listed()` gives the named cases, `draw(rng)` another one of the same ranges, `prepare(case, seed)` what a program holds
before the call, `run(state)` one pass (`own`: through the library, else in elementary torch operations in 32 bits),
`work(case)` the bytes and operations it cannot do without, `exact(case, seed)` the outputs in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6
BASE = 10000.0
BLOCK = 16                  # places of a page that share a power of two
LEAST, MOST = -48, 48       # its exponents
TOP = 448.0                 # the largest e4m3 number
WORKSPACE_BYTES = 64 << 20  # of the attention's key splits


# ----------------------------------------------------------------------------- the cases

def listed():
    return [
        # one decoded action token: 8 query heads on one key/value head, a layer's latency
        {"name": "store_decode_r1", "op": "store", "reqs": 1, "c_lo": 866, "c_hi": 866, "q_lo": 1, "q_hi": 1, "H": 8,
         "Hk": 1, "d": 128, "rot": 128, "pairs": "half", "axes": 1, "stretch": 1.0, "norm": True, "packed": False, "page": 16, "lens": 1},
        # drafted tokens of a batch: a few tokens each in the middle of begun blocks, image and text positions
        {"name": "store_drafts_r24_d64", "op": "store", "reqs": 24, "c_lo": 0, "c_hi": 3000, "q_lo": 1, "q_hi": 7, "H": 14,
         "Hk": 2, "d": 64, "rot": 64, "pairs": "half", "axes": 3, "stretch": 1.0, "norm": False, "packed": True, "page": 32, "lens": 2},
        # a decode batch far out in long contexts: neighbouring elements are pairs, half of a head turns, stretched
        {"name": "store_decode_r256", "op": "store", "reqs": 256, "c_lo": 100, "c_hi": 60000, "q_lo": 1, "q_hi": 1, "H": 32,
         "Hk": 8, "d": 128, "rot": 64, "pairs": "neighbours", "axes": 1, "stretch": 8.0, "norm": True, "packed": True, "page": 64, "lens": 3},
        # a prefill batch of a 2B backbone: heads of 256, prompts of ragged lengths
        {"name": "store_prefill_r12_d256", "op": "store", "reqs": 12, "c_lo": 0, "c_hi": 0, "q_lo": 700, "q_hi": 1900, "H": 8,
         "Hk": 1, "d": 256, "rot": 256, "pairs": "half", "axes": 1, "stretch": 1.0, "norm": False, "packed": False, "page": 64, "lens": 4},
        # one robot's prefix (3 x 256 image + 48 text tokens) out of the cache
        {"name": "read_prefix_816", "op": "read", "reqs": 1, "c_lo": 816, "c_hi": 816, "Hk": 1, "d": 128, "page": 16, "lens": 5},
        # the histories of a batch, to be moved or shared
        {"name": "read_r16_16k", "op": "read", "reqs": 16, "c_lo": 100, "c_hi": 16383, "Hk": 8, "d": 128, "page": 64, "lens": 6},
        # one decoded token over one robot's prefix and chunk: latency
        {"name": "attn_decode_r1", "op": "attn", "reqs": 1, "c_lo": 866, "c_hi": 866, "q_lo": 1, "q_hi": 1, "H": 8,
         "Hk": 1, "d": 128, "page": 16, "mask": "causal", "prefix": 0, "cap": 0.0, "window": 0, "lens": 7},
        # the action expert's 50-token chunk, all of it and the whole prefix visible
        {"name": "attn_chunk_m50", "op": "attn", "reqs": 1, "c_lo": 816, "c_hi": 816, "q_lo": 50, "q_hi": 50, "H": 8,
         "Hk": 1, "d": 128, "page": 16, "mask": "full", "prefix": 0, "cap": 0.0, "window": 0, "lens": 8},
        # a decode batch with ragged long histories: the cache's bandwidth
        {"name": "attn_decode_r64_16k", "op": "attn", "reqs": 64, "c_lo": 100, "c_hi": 16383, "q_lo": 1, "q_hi": 1,
         "H": 32, "Hk": 8, "d": 128, "page": 64, "mask": "causal", "prefix": 0, "cap": 0.0, "window": 0, "lens": 9},
        # drafted tokens checked in a batch: a few queries each, heads of 64, scores capped, sliding window
        {"name": "attn_drafts_r24_d64", "op": "attn", "reqs": 24, "c_lo": 0, "c_hi": 3000, "q_lo": 1, "q_hi": 7,
         "H": 14, "Hk": 2, "d": 64, "page": 32, "mask": "causal", "prefix": 0, "cap": 50.0, "window": 1024, "lens": 10},
        # a 2B backbone's prefill: heads of 256, the 768 image tokens visible to one another, the text causal
        {"name": "attn_prefix_m816_d256", "op": "attn", "reqs": 2, "c_lo": 0, "c_hi": 0, "q_lo": 816, "q_hi": 816,
         "H": 8, "Hk": 1, "d": 256, "page": 16, "mask": "prefix", "prefix": 768, "cap": 0.0, "window": 0, "lens": 11},
        # a chunk of a long prompt over what is cached already: the tensor cores' rate
        {"name": "attn_chunk_4096_of_16384", "op": "attn", "reqs": 1, "c_lo": 12288, "c_hi": 12288, "q_lo": 4096,
         "q_hi": 4096, "H": 32, "Hk": 8, "d": 128, "page": 64, "mask": "causal", "prefix": 0, "cap": 0.0,
         "window": 0, "lens": 12},
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _draw_once(rng):
    op = rng.choice(["store", "store", "read", "attn", "attn", "attn"])
    d = rng.choice([64, 128, 128, 256])
    Hk = rng.choice([1, 2, 4, 8])
    H = Hk * rng.choice([1, 2, 4, 7, 8])
    base = {"op": op, "Hk": Hk, "d": d, "page": rng.choice([16, 32, 64, 128]), "lens": rng.randrange(1 << 30)}
    if op == "read":
        return base | {"reqs": _log(rng, 1, 64), "c_lo": 1, "c_hi": _log(rng, 16, 16383)}
    kind = rng.choice(["decode", "drafts", "prefill"])
    reqs = rng.choice([1, _log(rng, 1, 64 if op == "attn" else 256)])
    q_hi = 1 if kind == "decode" else _log(rng, 2, 16) if kind == "drafts" else _log(rng, 16, 4096)
    base |= {"reqs": reqs, "q_lo": rng.choice([0, q_hi]) if reqs > 1 else q_hi, "q_hi": q_hi, "H": H}
    if op == "store":
        return base | {"c_lo": 0, "c_hi": rng.choice([0, _log(rng, 16, 60000)]), "rot": rng.choice([d, d, d // 2]),
                       "pairs": rng.choice(["half", "neighbours"]), "axes": rng.choice([1, 3]),
                       "stretch": rng.choice([1.0, 8.0]), "norm": rng.random() < 0.6, "packed": rng.random() < 0.5}
    c_hi = _log(rng, 16, 16000)
    return base | {"c_lo": rng.choice([0, c_hi // 2]), "c_hi": c_hi,
                   "mask": rng.choice(["causal", "causal", "prefix", "full"]), "prefix": _log(rng, 1, 1000),
                   "cap": rng.choice([0.0, 0.0, 30.0, 50.0]), "window": rng.choice([0, 0, 0, _log(rng, 1, 4096)])}


def _cost(case):
    """Seconds at the card's rates, and GB that the plain form's padded tensors take."""
    w = work(case)
    gb = 0.0
    if case["op"] == "attn":
        q, kv = _lengths(case)
        gb = 4e-9 * len(q) * max(kv) * (max(q) * case["H"] + 2 * case["Hk"] * case["d"])
    return w["bytes"] / 6.8e12 + w["flops"] / 1.9e15, gb


def draw(rng):
    """Another case of the listed ranges: sizes over their logarithm from one token to the largest listed ones, no
    costlier than the largest of its operator."""
    while True:
        case = _draw_once(rng)
        largest = [_cost(c) for c in listed() if c["op"] == case["op"]]
        if all(c <= max(x[i] for x in largest) for i, c in enumerate(_cost(case))):
            return case


def _lengths(case):
    """New and total tokens of every request."""
    r = random.Random(case["lens"])
    cached = [r.randint(case["c_lo"], case["c_hi"]) for _ in range(case["reqs"])]
    if case["op"] == "read":
        return [0] * case["reqs"], cached
    new = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["reqs"])]
    if sum(new) == 0:
        new[0] = 1
    return new, [c + n for c, n in zip(cached, new)]


def _range(case, p, kv, prefix):
    """Keys [lo, hi) that the query at position p sees."""
    return (max(0, p - case["window"] + 1) if case["window"] else 0), min(kv, max(p + 1, prefix))


def _prefix_of(case, kv):
    return {"causal": 0, "prefix": min(case["prefix"], kv), "full": kv}[case["mask"]]


def _frequencies(case):
    """Radians per position of a head's pairs: stretched, pairs that turn less than once in the context that the factors
    were made for keep to it (position / stretch), pairs that turn 32 times and more are left, in between by parts."""
    out = []
    for i in range(case["rot"] // 2):
        f = BASE ** (-2.0 * i / case["rot"])
        if case["stretch"] != 1.0:
            turns = 8192.0 * f / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
            f = f * (keep + (1.0 - keep) / case["stretch"])
        out.append(f)
    return out


# ----------------------------------------------------------------------------- inputs

def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _pages(kv, page, g, spare):
    """Pages in a random order of the cache: the block table (-1 past a request's pages)."""
    need = [-(-n // page) for n in kv]
    n_pages = sum(need) + spare
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    width = max(1, max(need))
    need_t = _ints(need, torch.int64)
    first = need_t.cumsum(0) - need_t
    col = torch.arange(width, device="cuda")[None]
    table = torch.where(col < need_t[:, None], perm[(first[:, None] + col).clamp(max=n_pages - 1)], -1).to(torch.int32)
    return table, n_pages


def _cache(n_pages, page, Hk, d, g):
    """Codes and exponents (plus 127) of normal values, as a store of whole blocks leaves them."""
    size = 1.0 + 3.0 * torch.rand(n_pages, page // BLOCK, 1, Hk, 1, generator=g, device="cuda")
    x = torch.randn(n_pages, page // BLOCK, BLOCK, Hk, d, generator=g, device="cuda") * size
    e = torch.ceil(torch.log2(x.abs().amax((2, 4), keepdim=True) / TOP))
    codes = (x * torch.exp2(-e)).clamp(-TOP, TOP).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.reshape(n_pages, page, Hk, d), (e + 127.0).to(torch.uint8).reshape(n_pages, page // BLOCK, Hk)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = {"device": "cuda"}

    def normal(*shape):
        return torch.randn(*shape, generator=g, **dev).to(torch.bfloat16)

    s = {"case": case}
    new, kv = _lengths(case)
    Hk, d, page = case["Hk"], case["d"], case["page"]
    op = case["op"]
    if op == "store":
        # the cache's pages are those of the step: of every request the page that it goes on with, and the new ones
        first = [(n - a) // page * page for n, a in zip(kv, new)]  # position of the first page
        table, n_pages = _pages([n - f for n, f in zip(kv, first)], page, g, 2)
        T = sum(new)
        req = torch.repeat_interleave(torch.arange(len(new), **dev), _ints(new, torch.int64))
        begin = _ints(new, torch.int64).cumsum(0) - _ints(new, torch.int64)
        in_req = torch.arange(T, **dev) - begin[req]
        pos = (_ints(kv, torch.int64) - _ints(new, torch.int64))[req] + in_req
        at = pos - _ints(first, torch.int64)[req]
        s["slots"] = table[req, at // page].long() * page + at % page
        H = case["H"]
        if case["packed"]:
            rows = normal(T, (H + 2 * Hk) * d)
            s["q"], s["k"], s["v"] = rows.split([H * d, Hk * d, Hk * d], dim=1)
        else:
            s["q"], s["k"], s["v"] = normal(T, H * d), normal(T, Hk * d), normal(T, Hk * d)
        gamma = 1.0 + 0.1 * torch.randn(2, d, generator=g, **dev)
        s["q_gamma"], s["k_gamma"] = (gamma[0], gamma[1]) if case["norm"] else (None, None)
        half = case["rot"] // 2
        if case["axes"] == 1:
            s["positions"], parts = pos.to(torch.int32)[None], [half]
        else:  # time, height and width of images of 16 x 16 tokens; a quarter of the pairs turns with time
            s["positions"] = torch.stack([pos // 256, pos // 256 + pos % 256 // 16, pos // 256 + pos % 16]).to(torch.int32)
            parts = [half // 4, half * 3 // 8, half - half // 4 - half * 3 // 8]
        s["axis_of_pair"] = None if case["axes"] == 1 else _ints([a for a, n in enumerate(parts) for _ in range(n)], torch.uint8)
        s["frequencies"] = torch.tensor(_frequencies(case), dtype=torch.float64, **dev)
        # turns a position in units of 2^-64
        s["turns"] = _ints([int(f / (2.0 * math.pi) * 2.0 ** 64) for f in _frequencies(case)], torch.int64)
        s["q_out"] = torch.empty(T, H * d, dtype=torch.bfloat16, **dev)
        # the places of every block that the step writes to
        s["all"] = (torch.unique(s["slots"] // BLOCK)[:, None] * BLOCK + torch.arange(BLOCK, **dev)).flatten()
    else:
        s["table"], n_pages = _pages(kv, page, g, 2)
    s["k_codes"], s["k_exp"] = _cache(n_pages, page, Hk, d, g)
    s["v_codes"], s["v_exp"] = _cache(n_pages, page, Hk, d, g)
    if op == "attn":
        s["q"] = normal(sum(new), case["H"] * d)
        start = [0]
        for n in new:
            start.append(start[-1] + n)
        s["q_start"], s["kv_len"], s["max_q"] = _ints(start), _ints(kv), max(new)
        s["prefix"] = None if case["mask"] == "causal" else _ints([_prefix_of(case, n) for n in kv])
        s["scale"] = d ** -0.5
        s["o"] = torch.empty(sum(new), case["H"] * d, dtype=torch.bfloat16, **dev)
        s["workspace"] = torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, **dev)
        return s
    if op == "read":
        req = torch.repeat_interleave(torch.arange(len(kv), **dev), _ints(kv, torch.int64))
        begin = _ints(kv, torch.int64).cumsum(0) - _ints(kv, torch.int64)
        at = torch.arange(sum(kv), **dev) - begin[req]
        s["all"] = s["table"][req, at // page].long() * page + at % page
    s["k_out"], s["v_out"] = (torch.empty(s["all"].shape[0], Hk * d, dtype=torch.bfloat16, **dev) for _ in range(2))
    return s


# ----------------------------------------------------------------------------- one pass

def run(state):
    if own:
        return {"store": _own_store, "read": _own_read, "attn": _own_attn}[state["case"]["op"]](state)
    return {"store": _plain_store, "read": _plain_read, "attn": _plain_attn}[state["case"]["op"]](state)


def _own_store(s):
    import paper_2607_02501_gb300 as emb
    emb.emb_paged8_store(s["q"], s["k"], s["v"], s["q_out"], s["k_codes"], s["v_codes"], s["k_exp"], s["v_exp"], s["slots"],
                         s["positions"], s["turns"], q_gamma=s["q_gamma"], k_gamma=s["k_gamma"], eps=EPS,
                         axis_of_pair=s["axis_of_pair"], neighbours=s["case"]["pairs"] == "neighbours")
    return {"q_out": s["q_out"], **_own_read(s)}  # and what the blocks hold now, as values


def _own_read(s):
    import paper_2607_02501_gb300 as emb
    emb.emb_paged8_read(s["k_codes"], s["v_codes"], s["k_exp"], s["v_exp"], s["all"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attn(s):
    import paper_2607_02501_gb300 as emb
    c = s["case"]
    emb.emb_paged8_attention(s["q"], s["k_codes"], s["v_codes"], s["k_exp"], s["v_exp"], s["table"], s["q_start"],
                             s["kv_len"], s["o"], s["scale"], s["max_q"], s["workspace"], prefix=s["prefix"], cap=c["cap"],
                             window=c["window"])
    return s["o"]


def _values(codes, exp):
    """What the cache holds, [pages][blocks][16][heads][d]."""
    n, page, Hk, d = codes.shape
    x = codes.view(torch.float8_e4m3fn).float().view(n, page // BLOCK, BLOCK, Hk, d)
    return x * torch.exp2(exp.float() - 127.0)[:, :, None, :, None]


def _plain_append(rows, codes, exp, slots):
    """fp32 rows [T][heads][d] into their slots."""
    n, page, Hk, d = codes.shape
    old = _values(codes, exp).view(-1, BLOCK, Hk, d)
    before = exp.float().view(-1, Hk) - 127.0
    top = torch.zeros(old.shape[0], BLOCK, Hk, device="cuda")
    top.view(-1, Hk)[slots] = rows.abs().amax(-1)
    written = torch.zeros(old.shape[0], BLOCK, dtype=torch.bool, device="cuda")
    written.view(-1)[slots] = True
    m, e = torch.frexp(top.amax(1) / TOP)  # the least power of two that takes the new rows
    need = torch.where(m == 0.5, e - 1, e).float().clamp(LEAST, MOST)
    need = torch.where(top.amax(1) > 0, need, float(LEAST))
    fresh = written[:, 0, None]  # a block whose first place is written starts anew
    after = torch.where(fresh, need, torch.maximum(before, need))
    after = torch.where(written.any(1)[:, None], after, before)
    x = torch.where(fresh[:, None, :, None], 0.0, old)
    x.view(-1, Hk, d)[slots] = rows
    x = x * torch.exp2(-after)[:, None, :, None]
    codes.copy_(x.to(torch.float8_e4m3fn).view(torch.uint8).view(n, page, Hk, d))
    exp.copy_((after + 127.0).to(torch.uint8).view(exp.shape))


def _plain_store(s):
    c = s["case"]
    H, Hk, d, rot = c["H"], c["Hk"], c["d"], c["rot"]
    T, half = s["q"].shape[0], c["rot"] // 2
    axis = torch.zeros(half, dtype=torch.int64, device="cuda") if s["axis_of_pair"] is None else s["axis_of_pair"].long()
    angle = s["positions"][axis].T.double() * s["frequencies"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x, heads, gamma):
        x = x.reshape(T, heads, d).float()
        if gamma is not None:
            x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * gamma
        if c["pairs"] == "half":
            a, b = x[..., :half], x[..., half:rot]
            return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
        a, b = x[..., :rot:2], x[..., 1:rot:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., rot:]], -1)

    s["q_out"].copy_(turned(s["q"], H, s["q_gamma"]).view(T, H * d))
    _plain_append(turned(s["k"], Hk, s["k_gamma"]), s["k_codes"], s["k_exp"], s["slots"])
    _plain_append(s["v"].reshape(T, Hk, d).float(), s["v_codes"], s["v_exp"], s["slots"])
    return {"q_out": s["q_out"], **_plain_read(s)}


def _plain_read(s):
    w = s["k_out"].shape[1]
    for name in ("k", "v"):
        s[name + "_out"].copy_(_values(s[name + "_codes"], s[name + "_exp"]).view(-1, w)[s["all"]])
    return {"k": s["k_out"], "v": s["v_out"]}


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

    def gathered(name):
        return _values(s[name + "_codes"][pages].view(-1, page, Hk, d), s[name + "_exp"][pages].view(-1, page // BLOCK, Hk)).view(R, L, Hk, d)

    x = (q @ gathered("k").permute(0, 2, 3, 1)).view(R, Hk, G, mq, L) * s["scale"]
    del q
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
    o = (x.view(R, Hk, G * mq, L) @ gathered("v").permute(0, 2, 1, 3)).view(R, Hk, G, mq, d) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(R, mq, H * d).to(torch.bfloat16)
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(start[1:], t, right=True)
    return o[r, t - start[r]]


# ----------------------------------------------------------------------------- what a pass needs

def work(case):
    Hk, d, page = case["Hk"], case["d"], case["page"]
    new, kv = _lengths(case)
    row = Hk * d  # bytes of a token's codes, keys or values
    if case["op"] == "read":
        n = sum(kv)
        return {"bytes": n * (2 * row + 4 * row + 8) + 2 * Hk * sum(-(-x // BLOCK) for x in kv), "flops": 2 * n * row}
    H = case["H"]
    if case["op"] == "store":
        T = sum(new)
        places = BLOCK * sum(-(-n // BLOCK) - (n - a) // BLOCK for n, a in zip(kv, new) if a > 0)
        # queries in and out, keys and values in, their codes out; what was there before in, all of it out as values
        return {"bytes": T * (4 * H * d + 4 * row + 2 * row + 8 + 4 * case["axes"]) + (places - T) * 2 * row + places * (4 * row + 8),
                "flops": T * (H + Hk) * d * (6 if case["norm"] else 3) + T * 4 * row}
    keys = blocks = pairs = 0
    for n, total in zip(new, kv):
        if n == 0:
            continue
        f = _prefix_of(case, total)
        spans = [_range(case, total - n + i, total, f) for i in range(n)]
        pairs += sum(max(0, hi - lo) for lo, hi in spans)
        lo, hi = min(lo for lo, _ in spans), max(hi for _, hi in spans)
        keys += hi - lo
        blocks += -(-hi // BLOCK) - lo // BLOCK
    return {"bytes": 4 * sum(new) * H * d + 2 * keys * row + 2 * blocks * Hk + 4 * keys // page + 8 * len(kv),
            "flops": 4 * pairs * H * d}


# ----------------------------------------------------------------------------- 64-bit outputs

def _rounded(x):
    """To the nearest e4m3 number, ties to the even one."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(x / step) * step


def _exact_values(codes, exp, page_of, place):
    """fp64 rows of the given places: the sign, exponent and mantissa of each code, times its block's power."""
    b = codes[page_of, place].long()
    e, m = b >> 3 & 15, b & 7
    x = torch.where(e > 0, (8 + m).double() * torch.exp2((e - 10).double()), m.double() * 2.0 ** -9)
    return torch.where(b > 127, -x, x) * torch.exp2(exp[page_of, place // BLOCK].double() - 127.0)[..., None]


def exact(case, seed):
    """The outputs in 64 bits: block by block, request by request, head by head."""
    s = prepare(case, seed)
    Hk, d, page = case["Hk"], case["d"], case["page"]
    if case["op"] != "attn":
        at = s["all"]  # (of a store: whole blocks, in rising order)
        held = {n: _exact_values(s[n + "_codes"], s[n + "_exp"], at // page, at % page) for n in ("k", "v")}
        if case["op"] == "read":
            return {n: x.reshape(-1, Hk * d) for n, x in held.items()}
        H, rot, half, T = case["H"], case["rot"], case["rot"] // 2, s["q"].shape[0]
        turn = torch.zeros(T, half, dtype=torch.float64, device="cuda")
        axes = [0] * half if s["axis_of_pair"] is None else s["axis_of_pair"].tolist()
        for i, f in enumerate(_frequencies(case)):
            turn[:, i] = s["positions"][axes[i]].double() * f
        spin = torch.polar(torch.ones_like(turn), turn)[:, None]
        first = torch.arange(half, device="cuda") * (1 if case["pairs"] == "half" else 2)
        second = first + (half if case["pairs"] == "half" else 1)
        rows = {"v": s["v"].reshape(T, Hk, d).double()}
        for name, heads, gamma in (("q", H, s["q_gamma"]), ("k", Hk, s["k_gamma"])):
            x = s[name].reshape(T, heads, d).double()
            if gamma is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS) * gamma.double()
            z = torch.complex(x[..., first], x[..., second]) * spin
            rows[name] = x.index_copy(-1, first, z.real).index_copy(-1, second, z.imag)
        slots = s["slots"].tolist()
        places = {}
        for t, slot in enumerate(slots):
            places.setdefault(slot // BLOCK, []).append((slot % BLOCK, t))
        exps = {n: s[n + "_exp"].reshape(-1, Hk).double() - 127.0 for n in ("k", "v")}
        row_of = {b: i * BLOCK for i, b in enumerate(sorted(places))}
        for block, got in places.items():
            p, t = _ints([x[0] for x in got], torch.int64), _ints([x[1] for x in got], torch.int64)
            for n in ("k", "v"):
                new = rows[n][t]
                e = torch.ceil(torch.log2(new.abs().amax((0, 2)) / TOP)).clamp(LEAST, MOST)
                mine = held[n][row_of[block]:row_of[block] + BLOCK]
                if any(x[0] == 0 for x in got):
                    mine.zero_()
                else:
                    e = torch.maximum(e, exps[n][block])
                mine[p] = new
                unit = torch.exp2(e)[None, :, None]
                mine.copy_(_rounded(mine / unit) * unit)
        return {"q_out": rows["q"].reshape(T, H * d), "k": held["k"].reshape(-1, Hk * d), "v": held["v"].reshape(-1, Hk * d)}
    new, kv = _lengths(case)
    H, G = case["H"], case["H"] // Hk
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
        k = _exact_values(s["k_codes"], s["k_exp"], page_of, idx % page)
        v = _exact_values(s["v_codes"], s["v_exp"], page_of, idx % page)
        for h in range(H):
            z = s["q"][at:at + n, h * d:(h + 1) * d].double() @ k[:, h // G].T * s["scale"]
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            z = torch.where(seen, z, -math.inf)
            w = torch.exp(z - z.amax(1, keepdim=True))
            out[at:at + n, h] = w @ v[:, h // G] / w.sum(1, keepdim=True)
        at += n
    return out.reshape(sum(new), H * d)
