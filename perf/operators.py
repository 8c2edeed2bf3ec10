"""The measured operators around the paged cache: what prepares a layer's query,
key and value rows for it, and decode attention that reads only the pages a cheap
score selects.

  norm_rope  a projection's fused rows -> queries and keys normalised per head and
             rotated by their positions (one axis, or time, height and width), values
             laid out beside them, in the layouts that the cache takes
  bounds     channelwise least and largest key of each page, per layer and KV head
  scores     for every page, the largest logit that any of a KV head's queries could
             have on one of its tokens, from the bounds
  top        the pages that a decode step attends: the first, the last, and those of the
             highest scores, in the order of the sequence
  attend     attention of one new token per sequence over selected pages, and the mass
             that each of their tokens received

`run` computes an operator by elementary torch operations in 32 bits, or, where `own`
is true, by the library.

Fields of a case:
  op       one of the above
  layers, q_heads, kv_heads, page   attention geometry, tokens per page
  batch, tokens, ragged, empty   sequences, tokens of the longest, the share by which the
           others may be shorter, whether the last one holds no token (page operators)
  top      pages that are kept per row ("top", "attend")
  closed   only the last page of each sequence is bounded, as when decode steps filled it
  mass     the masses are written as well ("attend")
  tokens, type, axes, rotary, interleaved, norm   rows, their type, position axes, rotated
           channels, pairs (2i, 2i+1) instead of (i, i + rotary/2), head norms ("norm_rope")

Keys, values and queries are N(0, 1), with a few tokens attended more strongly along one
direction.  Slots past a sequence's tokens hold NaN: nothing may read them into a result."""
import math
import random

import numpy as np
import torch

own = False

D = 128
EPS = 1e-6
ROPE_BASE = 1e6
HOT_DIMS, HOT_KEY, HOT_QUERY, HOT_SHARE = 16, 2.0, 0.5, 0.02
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

DEFAULTS = {"op": "attend", "layers": 1, "q_heads": 16, "kv_heads": 2, "page": 16, "batch": 1, "tokens": 1700,
            "ragged": 0.0, "empty": False, "top": 0, "closed": False, "mass": False, "type": "bf16", "axes": 1,
            "rotary": D, "interleaved": False, "norm": True}


def _case(name, **kw):
    c = dict(DEFAULTS, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one agent's new token in one layer, 1.5B geometry: the shortest call of a decode loop
        _case("norm_rope 1 token", op="norm_rope", q_heads=12, tokens=1),
        # a serving batch's new tokens, kept in 32 bits by the projection, with image positions
        _case("norm_rope 32 tokens f32 3 axes", op="norm_rope", tokens=32, type="f32", axes=3),
        # one layer of a long prompt on its way into the cache, 3B geometry
        _case("norm_rope 8191 tokens", op="norm_rope", tokens=8191),
        # 32 sequences have each filled a page: bounded before the next step selects
        _case("bounds 32 pages L36", op="bounds", layers=36, batch=32, tokens=1700, ragged=0.5, closed=True),
        # a long prompt was appended: all of its pages, all layers
        _case("bounds 1x8192 L36", op="bounds", layers=36, tokens=8192),
        # one agent's history, one layer
        _case("scores 1x32768 L1", op="scores", tokens=32768),
        # eight long histories, all layers at once
        _case("scores 8x131072 L36 p32", op="scores", layers=36, page=32, batch=8, tokens=131072, ragged=0.2),
        # the selection of that layer call
        _case("top 1x32768 L1", op="top", tokens=32768, top=64),
        # the selection of that step
        _case("top 8x131072 L36 p32", op="top", layers=36, page=32, batch=8, tokens=131072, ragged=0.2, top=64),
        # one agent, one layer: the selected pages of its history
        _case("attend 1x32768 L1", op="attend", tokens=32768, top=64, mass=True),
        # a serving batch's layer, short and empty sequences among it
        _case("attend 32x8000 L1", op="attend", batch=32, tokens=8000, ragged=0.95, empty=True, top=48, mass=True),
        # long histories, all layers at once: the largest call
        _case("attend 4x65536 L36 p32", op="attend", layers=36, page=32, batch=4, tokens=65536, ragged=0.2, top=128,
              mass=True),
    ]


MAX_BYTES = 1.3e9          # the largest listed case's work
MAX_POOL = 1.0e10          # K/V held by a state


def _log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n + 1 if n > 512 and n % 512 == 0 else n     # a trace's length is not round


def draw(rng):
    while True:
        q_heads, kv_heads = rng.choice(((12, 2), (16, 2), (16, 2), (8, 2), (8, 1), (28, 4), (32, 8)))
        op = rng.choice(("norm_rope", "norm_rope", "bounds", "scores", "top", "attend", "attend", "attend"))
        c = _case("", op=op, q_heads=q_heads, kv_heads=kv_heads)
        if op == "norm_rope":
            c.update(tokens=_log_int(rng, 1, 40000), type=rng.choice(("bf16", "bf16", "f16", "f32")),
                     axes=rng.choice((1, 1, 3)), rotary=rng.choice((128, 128, 64, 32)),
                     interleaved=rng.random() < 0.3, norm=rng.random() < 0.7)
        else:
            c.update(layers=rng.choice((1, 1, 1, 2, 4, 8, 16, 28, 36)), page=rng.choice((16, 32)),
                     batch=_log_int(rng, 1, 64), tokens=_log_int(rng, 1, 131072),
                     ragged=rng.choice((0.0, 0.3, 0.8, 0.95)))
            c["empty"] = c["batch"] > 1 and rng.random() < 0.3
            if op in ("top", "attend"):
                c["top"] = _log_int(rng, 4 if op == "top" else 2, 300)
            if op == "top" and c["tokens"] < 2 * c["top"] * c["page"]:
                continue                                # the longest sequence has something to leave out
            if op == "bounds":
                c["closed"] = rng.random() < 0.3
            if op == "attend":
                c["mass"] = rng.random() < 0.5
        if work(c)["bytes"] <= MAX_BYTES and _pool_bytes(c) <= MAX_POOL:
            return c


# ------------------------------------------------------------------ shapes ----
def _lengths(c):
    """Tokens per sequence (the same for every seed)."""
    r = random.Random(c["batch"] * 1000003 + c["tokens"])
    n = [max(1, int(c["tokens"] * (1.0 - (c["ragged"] * r.random() if b else 0.0)))) for b in range(c["batch"])]
    if c["empty"]:
        n[-1] = 0
    return n


def _pages(c):
    return [-(-n // c["page"]) for n in _lengths(c)]


def _pool_bytes(c):
    if c["op"] in ("norm_rope", "top"):
        return 0
    per_page = 4 * D * (c["page"] if c["op"] != "scores" else 1)
    return sum(_pages(c)) * c["layers"] * c["kv_heads"] * per_page


def work(case):
    """Each input once and each output once: rows, positions and table rows in and bf16
    rows out; the keys of the bounded pages in and their bounds out; bounds and queries in
    and scores out; scores in and page numbers out; the selected pages' K and V, the
    queries and page numbers in, outputs and masses out."""
    c = dict(DEFAULTS, **case)
    Hq, Hkv, L, page, op = c["q_heads"], c["kv_heads"], c["layers"], c["page"], c["op"]
    if op == "norm_rope":
        T, rows = c["tokens"], c["q_heads"] + 2 * c["kv_heads"]
        size = 4 if c["type"] == "f32" else 2
        return {"bytes": T * (rows * D * (size + 2) + c["axes"] * 4 + c["rotary"] * 4), "flops": T * (Hq + Hkv) * D * 7}
    n, p, items = _lengths(c), _pages(c), L * Hkv
    q_bytes = c["batch"] * L * Hq * D * 2
    if op == "bounds":
        keys = sum((x - 1) % page + 1 for x in n if x) if c["closed"] else sum(n)
        done = sum(1 for x in n if x) if c["closed"] else sum(p)
        return {"bytes": items * (keys * 2 * D + done * 4 * D), "flops": items * keys * 2 * D}
    if op == "scores":
        return {"bytes": sum(p) * items * (4 * D + 4) + q_bytes, "flops": sum(p) * L * Hq * 4 * D}
    if op == "top":
        return {"bytes": items * (sum(p) * 4 + c["batch"] * c["top"] * 4), "flops": sum(p) * items}
    kept = sum(min(x, c["top"]) for x in p)
    tokens = sum(min(x, c["top"]) * page - (-y % page) for x, y in zip(p, n) if x)
    mass = 4 * c["batch"] * items * c["top"] * page if c["mass"] else 0
    return {"bytes": items * (tokens * 4 * D + kept * 4) + 2 * q_bytes + mass, "flops": 4 * Hq * D * L * tokens}


# ------------------------------------------------------------------- state ----
def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + what) % (1 << 61))
    return g


def _axis_of_pair(c):
    """The position axis of each rotated pair: time, height and width in turn, what is left over to time."""
    n = c["rotary"] // 2
    if c["axes"] == 1:
        return np.zeros(n, np.uint8)
    each = n // 3
    return np.array([i % 3 if i < 3 * each else 0 for i in range(n)], np.uint8)


def _positions(c, seed):
    """int32 [axes][tokens]: decode tokens of many sequences lie anywhere, a prompt's follow each
    other; with three axes, images of 24 x 18 patches stand in it."""
    T, g = c["tokens"], _gen(seed, 3)
    if T <= 64:
        return torch.randint(0, 32768, (c["axes"], T), generator=g, device="cuda", dtype=torch.int32)
    start = int(torch.randint(0, 1000, (1,), generator=g, device="cuda"))
    t = torch.arange(T, device="cuda", dtype=torch.int32)
    if c["axes"] == 1:
        return (t + start)[None]
    return torch.stack([t // 432 + start, t % 432 // 24 + start, t % 24 + start]).contiguous()


def _inv_freq(c):
    n = c["rotary"] // 2
    return torch.exp(torch.arange(n, dtype=torch.float64, device="cuda") * (-math.log(ROPE_BASE) / n))


def _prepare_norm_rope(c, seed):
    T, Hq, Hkv, R = c["tokens"], c["q_heads"], c["kv_heads"], c["rotary"]
    g = _gen(seed, 1)
    rows = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device="cuda", dtype=TYPES[c["type"]])
    weight = 1.0 + 0.2 * torch.randn((2, D), generator=g, device="cuda")
    pos = _positions(c, seed)
    length = max(32768, T + 1000)
    angle = torch.arange(length, dtype=torch.float64, device="cuda")[:, None] * _inv_freq(c)
    # a prompt's keys and values go to the cache as [kv_heads][tokens][D], decode tokens' as [tokens][kv_heads][D]
    lead = (T, Hkv, D) if T <= 64 else (Hkv, T, D)
    k, v = (torch.empty(lead, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if T > 64:
        k, v = k.transpose(0, 1), v.transpose(0, 1)
    return {"case": c, "q": rows[:, :Hq], "k": rows[:, Hq:Hq + Hkv], "v": rows[:, Hq + Hkv:], "positions": pos,
            "q_weight": weight[0] if c["norm"] else None, "k_weight": weight[1] if c["norm"] else None,
            "table": torch.stack([torch.cos(angle), torch.sin(angle)], -1).float(), "axes": _axis_of_pair(c),
            "axes_dev": torch.from_numpy(_axis_of_pair(c)).cuda().long(),
            "q_out": torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda"), "k_out": k, "v_out": v}


def _table(c, seed):
    """The block table (an engine's pages lie anywhere in its pool) and the pages in the pool."""
    pages = _pages(c)
    ids = list(range(max(1, sum(pages))))
    random.Random(seed).shuffle(ids)
    table = np.zeros((c["batch"], max(1, max(pages))), np.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = ids[at:at + p]
        at += p
    return torch.from_numpy(table).cuda(), len(ids)


def _pool(c, seed, table, P):
    L, Hkv, page = c["layers"], c["kv_heads"], c["page"]
    pool = torch.empty((L, P, Hkv, 2, page, D), dtype=torch.bfloat16, device="cuda")
    pool.normal_(generator=_gen(seed, 4))
    hot = torch.rand((P, page), generator=_gen(seed, 5), device="cuda") < HOT_SHARE
    pool[:, :, :, 0, :, :HOT_DIMS] += (HOT_KEY * hot)[None, :, None, :, None].to(torch.bfloat16)
    for b, n in enumerate(_lengths(c)):
        if n % page:
            pool[:, int(table[b, n // page]), :, :, n % page:] = math.nan
    return pool


def _queries(c, seed):
    q = torch.randn((c["batch"], c["layers"], c["q_heads"], D), generator=_gen(seed, 6), device="cuda",
                    dtype=torch.bfloat16)
    q[..., :HOT_DIMS] += HOT_QUERY
    return q


def _pick(c, seed):
    """Selected pages int32 [batch][layers][kv_heads][top], in order, -1 behind them: the first
    and the last of each sequence and others at random."""
    lead, most = (c["batch"], c["layers"], c["kv_heads"]), max(1, max(_pages(c)))
    n = torch.tensor(_pages(c), device="cuda").view(-1, 1, 1, 1)
    at = torch.arange(most, device="cuda")
    key = torch.rand(lead + (most,), generator=_gen(seed, 7), device="cuda")
    key = torch.where((at == 0) | (at == n - 1), 2.0, key).masked_fill(at >= n, -1.0)
    val, idx = key.topk(min(most, c["top"]), -1)
    idx = torch.where(val >= 0, idx, 1 << 30).sort(-1).values
    out = torch.full(lead + (c["top"],), -1, dtype=torch.int32, device="cuda")
    out[..., :idx.shape[-1]] = torch.where(idx < 1 << 30, idx, -1).int()
    return out


def prepare(case, seed):
    c = dict(DEFAULTS, **case)
    op = c["op"]
    if op == "norm_rope":
        return _prepare_norm_rope(c, seed)
    lead, most = (c["batch"], c["layers"], c["kv_heads"]), max(1, max(_pages(c)))
    s = {"case": c, "tokens": np.array(_lengths(c), np.int32)}
    s["tokens_dev"] = torch.from_numpy(s["tokens"]).cuda().long()
    s["pages_dev"] = (s["tokens_dev"] + c["page"] - 1) // c["page"]
    if op == "top":
        # the bounds of a page's logits; agents that share a prompt have pages of equal scores
        x = 3.0 + torch.randn(lead + (most,), generator=_gen(seed, 8), device="cuda")
        x[..., 1::3] = x[..., 0:most - 1:3]
        s["scores"] = x.masked_fill(torch.arange(most, device="cuda") >= s["pages_dev"].view(-1, 1, 1, 1), math.nan)
        s["out"] = torch.empty(lead + (c["top"],), dtype=torch.int32, device="cuda")
        return s
    s["table"], P = _table(c, seed)
    shape = (c["layers"], P, c["kv_heads"], 2, D)
    if op == "scores":
        mid = torch.randn(shape, generator=_gen(seed, 9), device="cuda", dtype=torch.bfloat16) * 0.5
        mid[..., 0, :] -= 1.8
        mid[..., 1, :] += 1.8
        lo, hi = torch.minimum(mid[..., 0, :], mid[..., 1, :]), torch.maximum(mid[..., 0, :], mid[..., 1, :])
        s["bounds"] = torch.stack([lo, hi], -2)
        s["q"] = _queries(c, seed)
        s["out"] = torch.zeros(lead + (most,), device="cuda")
        return s
    s["pool"] = _pool(c, seed, s["table"], P)
    if op == "bounds":
        s["bounds"] = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        s["first"] = np.array([max(0, p - 1) if c["closed"] else 0 for p in _pages(c)], np.int32)
        s["first_dev"] = torch.from_numpy(s["first"]).cuda().long()
        return s
    s["q"], s["ids"] = _queries(c, seed), _pick(c, seed)
    s["out"] = torch.empty_like(s["q"])
    s["mass"] = torch.empty(lead + (c["top"] * c["page"],), device="cuda") if c["mass"] else None
    return s


# -------------------------------------------------------------- plain forms ----
def _plain_norm_rope(s):
    c, R = s["case"], s["case"]["rotary"]
    pair = torch.arange(R // 2, device="cuda")
    cs = s["table"][s["positions"][s["axes_dev"]].long().t(), pair][:, None]          # [T][1][R/2][2]

    def rows(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight
        a, b = (x[..., 0:R:2], x[..., 1:R:2]) if c["interleaved"] else (x[..., :R // 2], x[..., R // 2:R])
        a, b = a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]
        r = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
        return torch.cat([r, x[..., R:]], -1).bfloat16()

    return {"q": rows(s["q"], s["q_weight"]), "k": rows(s["k"], s["k_weight"]), "v": s["v"].float().bfloat16()}


def _plain_bounds(s):
    c = s["case"]
    page, at = c["page"], torch.arange(s["table"].shape[1], device="cuda")
    todo = (at >= s["first_dev"][:, None]) & (at < s["pages_dev"][:, None])
    b, p = todo.nonzero(as_tuple=True)
    phys = s["table"][b, p].long()
    k = s["pool"][:, phys, :, 0].float()                                              # [L][n][Hkv][page][D]
    held = (p[:, None] * page + torch.arange(page, device="cuda") < s["tokens_dev"][b][:, None])[None, :, None, :, None]
    s["bounds"][:, phys, :, 0] = torch.where(held, k, math.inf).amin(-2).bfloat16()
    s["bounds"][:, phys, :, 1] = torch.where(held, k, -math.inf).amax(-2).bfloat16()
    return {"bounds": s["bounds"]}


def _plain_scores(s):
    c = s["case"]
    B, L, Hkv = c["batch"], c["layers"], c["kv_heads"]
    at = torch.arange(s["table"].shape[1], device="cuda")
    x = s["bounds"][:, s["table"].long()].permute(1, 0, 3, 2, 4, 5).float()           # [B][L][Hkv][pages][2][D]
    q = s["q"].float().view(B, L, Hkv, -1, D)
    up = torch.matmul(x[..., 1, :], q.clamp(min=0).transpose(-1, -2))
    up += torch.matmul(x[..., 0, :], q.clamp(max=0).transpose(-1, -2))
    r = up.amax(-1) * (1.0 / math.sqrt(D))
    s["out"].copy_(torch.where(at < s["pages_dev"].view(-1, 1, 1, 1), r, s["out"]))
    return {"scores": s["out"]}


def _plain_top(s):
    c, x, n = s["case"], s["scores"], s["pages_dev"].view(-1, 1, 1, 1)
    most, top = x.shape[-1], c["top"]
    at = torch.arange(most, device="cuda")
    key = torch.where(x.isnan(), math.inf, x)
    key = torch.where((at == 0) | (at == n - 1), math.inf, key)
    key = key.masked_fill(at >= n, -math.inf)
    order = key.sort(dim=-1, descending=True, stable=True).indices[..., :top]
    order = torch.where(order < n, order, 1 << 30).sort(-1).values
    s["out"].fill_(-1)
    s["out"][..., :order.shape[-1]] = torch.where(order < 1 << 30, order, -1).int()
    return {"ids": s["out"]}


def _plain_attend(s):
    c = s["case"]
    B, L, Hkv, page = c["batch"], c["layers"], c["kv_heads"], c["page"]
    ids = s["ids"].long()
    here = ids >= 0
    phys = s["table"][torch.arange(B, device="cuda").view(-1, 1, 1, 1), ids.clamp(min=0)].long()
    layer = torch.arange(L, device="cuda").view(-1, 1, 1)
    head = torch.arange(Hkv, device="cuda").view(-1, 1)
    kv = s["pool"][layer, phys, head]                                                 # [B][L][Hkv][top][2][page][D]
    tok = ids[..., None] * page + torch.arange(page, device="cuda")
    held = (here[..., None] & (tok < s["tokens_dev"].view(-1, 1, 1, 1, 1))).flatten(-2)
    k = kv[..., 0, :, :].flatten(-3, -2).float()
    v = torch.where(held[..., None], kv[..., 1, :, :].flatten(-3, -2), 0).float()
    q = s["q"].float().view(B, L, Hkv, -1, D)
    x = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    x = torch.where(held[..., None, :], x, -math.inf)
    e = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e30))
    z = e.sum(-1, keepdim=True)
    p = torch.where(z > 0, e / z, 0.0)
    r = {"out": torch.matmul(p, v).view(B, L, -1, D).bfloat16()}
    if c["mass"]:
        r["mass"] = p.sum(-2)
    return r


# --------------------------------------------------------------- the library ----
def _own(s):
    import paper_2607_10582_gb300 as md
    c, op = s["case"], s["case"]["op"]
    if op == "norm_rope":
        md.md_norm_rope(s["q"], s["k"], s["v"], s["q_out"], s["k_out"], s["v_out"], positions=s["positions"],
                        table=s["table"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, axes=s["axes"],
                        interleaved=c["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if op == "bounds":
        md.md_page_bounds(s["pool"], s["table"], s["tokens"], s["bounds"], first_pages=s["first"])
        return {"bounds": s["bounds"]}
    if op == "scores":
        md.md_page_scores(s["q"], s["bounds"], s["table"], s["tokens"], s["out"], page_size=c["page"])
        return {"scores": s["out"]}
    if op == "top":
        md.md_page_top(s["scores"], s["tokens"], s["out"], page_size=c["page"], first=1, last=1)
        return {"ids": s["out"]}
    md.md_attend_pages(s["q"], s["pool"], s["table"], s["tokens"], s["ids"], s["out"], mass=s["mass"])
    return {"out": s["out"], "mass": s["mass"]} if c["mass"] else {"out": s["out"]}


def run(state):
    if own:
        return _own(state)
    return {"norm_rope": _plain_norm_rope, "bounds": _plain_bounds, "scores": _plain_scores, "top": _plain_top,
            "attend": _plain_attend}[state["case"]["op"]](state)


# ------------------------------------------------------------------- exact ----
def _exact_norm_rope(c, s):
    R, pos = c["rotary"], s["positions"].double()
    angle = torch.stack([pos[a] * f for a, f in zip(_axis_of_pair(c), _inv_freq(c))], -1)    # [T][R/2]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    first = torch.arange(R // 2, device="cuda")
    first, second = (2 * first, 2 * first + 1) if c["interleaved"] else (first, first + R // 2)
    r = {"v": s["v"].double()}
    for name in ("q", "k"):
        x = s[name].double()
        if c["norm"]:
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / D + EPS) * s[name + "_weight"].double()
        y = x.clone()
        z = torch.complex(x[..., first], x[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        r[name] = y
    return r


def exact(case, seed):
    """From the definitions, sequence by sequence and in 64 bits."""
    c = dict(DEFAULTS, **case)
    s = prepare(c, seed)
    op, page, L, Hkv, G = c["op"], c["page"], c["layers"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    if op == "norm_rope":
        return _exact_norm_rope(c, s)
    n, pages = _lengths(c), _pages(c)
    if op == "top":
        return None                  # page numbers only
    if op == "bounds":
        r = s["bounds"].double()
        for b in range(c["batch"]):
            full = pages[b] - (1 if n[b] % page else 0)
            for lo, hi, held in ((int(s["first"][b]), full, page), (max(full, int(s["first"][b])), pages[b], n[b] % page)):
                if lo < hi:
                    at = s["table"][b, lo:hi].long()
                    keys = s["pool"][:, at, :, 0, :held].double()
                    r[:, at, :, 0], r[:, at, :, 1] = keys.min(-2).values, keys.max(-2).values
        return {"bounds": r}
    if op == "scores":
        r = s["out"].double()
        for b in range(c["batch"]):
            for l in range(L):
                x = s["bounds"][l, s["table"][b, :pages[b]].long()].double()                  # [pages][Hkv][2][D]
                for h in range(Hkv):
                    q = s["q"][b, l, h * G:(h + 1) * G].double()
                    up = torch.where(q > 0, q, 0) @ x[:, h, 1].T + torch.where(q < 0, q, 0) @ x[:, h, 0].T
                    r[b, l, h, :pages[b]] = up.max(0).values / math.sqrt(D)
        return {"scores": r}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    mass = torch.zeros((c["batch"], L, Hkv, c["top"], page), dtype=torch.float64, device="cuda")
    offset, head = torch.arange(page, device="cuda"), torch.arange(Hkv, device="cuda")[:, None]
    for b in range(c["batch"]):
        m = min(pages[b], c["top"])
        for l in range(L if m else 0):
            ids = s["ids"][b, l, :, :m].long()
            kv = s["pool"][l, s["table"][b, ids].long(), head].double()                       # [Hkv][m][2][page][D]
            gone = (ids[..., None] * page + offset >= n[b]).flatten(1)
            k, v = (kv[:, :, i].flatten(1, 2).masked_fill(gone[..., None], 0) for i in (0, 1))
            x = torch.einsum("hgd,hnd->hgn", s["q"][b, l].double().view(Hkv, G, D), k) / math.sqrt(D)
            p = torch.softmax(x.masked_fill(gone[:, None], -math.inf), -1)
            out[b, l] = torch.einsum("hgn,hnd->hgd", p, v).flatten(0, 1)
            mass[b, l, :, :m] = p.sum(1).view(Hkv, m, page)
    return {"out": out, "mass": mass.flatten(3)} if c["mass"] else {"out": out}
