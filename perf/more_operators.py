"""The measured operators of a cache held in eight bits, and of attention over a whole cache
under a sliding window.

  write   new tokens' key and value rows -> their places in the pages of an e4m3 cache, with
          a scale (a power of two) for each 16 tokens of a layer, KV head, and K or V; a block
          that held tokens before keeps its scale, or, where the new ones exceed it, takes
          a larger one, and its older codes with it
  read    tokens of the cache -> rows again
  attend  attention of one new token per sequence over the cached tokens that its window shows
          (the last `window` ones, and the first `sinks` ones), of a cache in e4m3 or in bf16,
          and the logarithm of each head's sum of exponentials

`run` computes an operator by elementary torch operations in 32 bits, or, where `own`
is true, by the library.

Fields of a case:
  op       one of the above
  layers, q_heads, kv_heads, page   attention geometry, tokens per page
  batch, tokens, ragged, empty   sequences, tokens of the longest, the share by which the
           others may be shorter, whether the last one holds no token
  step     the last token of each sequence is written, the others are there; else all are new ("write")
  type     of the rows ("write", "read") or of the cache ("attend")
  window, sinks   of the attention; window -1: all tokens are visible

Keys, values and queries are N(0, 1), the keys and queries with a few strong channels, keys of a few
tokens stronger along one direction.  Slots that hold no token hold NaN where attention might read them."""
import math
import random

import numpy as np
import torch

own = False

D = 128
BLOCK = 16                 # tokens of a scale
MOST = 448.0               # largest e4m3 value
WORKSPACE = 1 << 24        # bytes that the attention may use
HOT_DIMS, HOT_KEY, HOT_QUERY, HOT_SHARE = 16, 2.0, 0.5, 0.02
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}

DEFAULTS = {"op": "attend", "layers": 1, "q_heads": 16, "kv_heads": 2, "page": 16, "batch": 1, "tokens": 1700,
            "ragged": 0.0, "empty": False, "step": False, "type": "e4m3", "window": -1, "sinks": 0}


def _case(name, **kw):
    c = dict(DEFAULTS, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one agent's new token in one layer: the shortest call of a decode loop
        _case("write 1 token L1", op="write", tokens=1001, step=True, type="bf16"),
        # a serving batch's step, all layers at once
        _case("write 32 tokens L36", op="write", layers=36, batch=32, tokens=1700, ragged=0.5, step=True, type="bf16"),
        # a long prompt on its way into the cache
        _case("write 8191 tokens L36", op="write", layers=36, tokens=8191, type="bf16"),
        # a tool's output of one agent, taken back in 32 bits by a layer that works on it
        _case("read 777 tokens L1 f32", op="read", tokens=777, type="f32"),
        # histories go back into a cache of 16 bits
        _case("read 4x4000 L36", op="read", layers=36, batch=4, tokens=4000, ragged=0.3, type="bf16"),
        # one agent, one layer, short history: latency
        _case("attend 1x448 L1", q_heads=12, tokens=448),
        # one agent's whole history, one layer: few rows, long
        _case("attend 1x131071 L1", tokens=131071),
        # a serving batch's layer, short and empty sequences among it, more KV heads
        _case("attend 32x8000 L1 Hkv 8", q_heads=32, kv_heads=8, batch=32, tokens=8000, ragged=0.95, empty=True),
        # a serving batch, all layers at once
        _case("attend 32x1700 L36", layers=36, batch=32, tokens=1700, ragged=0.5),
        # long histories, all layers at once: the largest call
        _case("attend 4x65536 L36 p32", layers=36, page=32, batch=4, tokens=65536, ragged=0.2),
        # a layer of a model with a sliding window, sinks kept, cache in eight bits
        _case("attend 16x13001 L1 window 4096", page=32, batch=16, tokens=13001, ragged=0.5, window=4096, sinks=4),
        # several such layers over a cache in bf16
        _case("attend bf16 8x32768 L4 window 1000", layers=4, batch=8, tokens=32768, ragged=0.3, window=1000, sinks=16,
              type="bf16"),
    ]


MAX_BYTES = 4.0e9          # the largest listed case's work
MAX_POOL = 6.0e9           # K/V held by a state


def _log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n + 1 if n > 512 and n % 512 == 0 else n     # a trace's length is not round


def draw(rng):
    while True:
        q_heads, kv_heads = rng.choice(((12, 2), (16, 2), (16, 2), (8, 2), (8, 1), (28, 4), (32, 8), (4, 4)))
        op = rng.choice(("write", "write", "read", "attend", "attend", "attend", "attend"))
        c = _case("", op=op, q_heads=q_heads, kv_heads=kv_heads, layers=rng.choice((1, 1, 1, 2, 4, 8, 16, 28, 36)),
                  page=rng.choice((16, 32)), batch=_log_int(rng, 1, 64), tokens=_log_int(rng, 1, 131072),
                  ragged=rng.choice((0.0, 0.3, 0.8, 0.95)))
        c["empty"] = c["batch"] > 1 and rng.random() < 0.3
        if op == "attend":
            c["type"] = rng.choice(("e4m3", "e4m3", "e4m3", "bf16"))
            if rng.random() < 0.4:
                c.update(window=_log_int(rng, 1, 16384), sinks=rng.choice((0, 0, 1, 4, 16, 33)))
        else:
            c["type"] = rng.choice(("bf16", "bf16", "f16", "f32"))
            c["step"] = op == "write" and rng.random() < 0.5
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
    return sum(_pages(c)) * c["page"] * c["layers"] * c["kv_heads"] * 2 * D * (2 if c["type"] == "bf16" and c["op"] == "attend" else 1)


def _spans(c):
    """Tokens that a write or a read is about: first, count, per sequence."""
    return [(n - 1, 1) if c["step"] and n else (0, n) for n in _lengths(c)]


def _shown(c, n):
    """A sequence's visible tokens: so many first ones, and all from a place on."""
    w0 = max(0, n - c["window"]) if c["window"] >= 0 else 0
    return min(c["sinks"], w0), w0


def _blocks(c):
    """Scales that a write or an attention meets, per layer, KV head, and K or V."""
    if c["op"] != "attend":
        return sum((a + n - 1) // BLOCK - a // BLOCK + 1 for a, n in _spans(c) if n)
    return sum((-(-s // BLOCK)) + -(-n // BLOCK) - w0 // BLOCK for n in _lengths(c) for s, w0 in (_shown(c, n),))


def work(case):
    """Each input once and each output once: rows in, codes and scales out; the other way round;
    visible codes (or bf16 values) and their scales, queries in, outputs and logarithms out."""
    c = dict(DEFAULTS, **case)
    Hq, L, items = c["q_heads"], c["layers"], c["layers"] * c["kv_heads"]
    if c["op"] != "attend":
        T = sum(n for _, n in _spans(c))
        size = 4 if c["type"] == "f32" else 2
        return {"bytes": items * 2 * (T * D * (size + 1) + _blocks(c) * 4), "flops": items * 2 * T * D * 2}
    tokens = sum(s + n - w0 for n in _lengths(c) for s, w0 in (_shown(c, n),))
    kv = tokens * 4 * D if c["type"] == "bf16" else tokens * 2 * D + _blocks(c) * 8
    return {"bytes": items * kv + c["batch"] * L * Hq * (4 * D + 4), "flops": 4 * Hq * D * L * tokens}


# ------------------------------------------------------------------- state ----
def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + what) % (1 << 61))
    return g


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


def _channels(seed):
    """Sizes of the channels of keys and queries: a few are strong."""
    return 1.0 + 3.0 * (torch.rand((D,), generator=_gen(seed, 2), device="cuda") < 0.04)


def _pool(c, seed, table, P):
    """A cache in bf16, NaN behind each sequence's tokens."""
    L, Hkv, page = c["layers"], c["kv_heads"], c["page"]
    pool = torch.empty((L, P, Hkv, 2, page, D), dtype=torch.bfloat16, device="cuda")
    pool.normal_(generator=_gen(seed, 4))
    pool[:, :, :, 0] *= _channels(seed).bfloat16()
    hot = torch.rand((P, page), generator=_gen(seed, 5), device="cuda") < HOT_SHARE
    pool[:, :, :, 0, :, :HOT_DIMS] += (HOT_KEY * hot)[None, :, None, :, None].to(torch.bfloat16)
    for b, n in enumerate(_lengths(c)):
        if n % page:
            pool[:, int(table[b, n // page]), :, :, n % page:] = math.nan
    return pool


def _power(e):
    """2^e in 32 bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _scale_of(most):
    """The least power of two s with most <= 448 s, and at least 2^-126."""
    part, e = torch.frexp(most)
    e = torch.where(most > 0, e - 9 + (part > MOST / 512), -126).clamp(min=-126)
    return _power(e)


def _quantised(pool):
    """(codes, scales) of a cache in bf16, layer by layer: NaN slots stay NaN."""
    L, P, Hkv, _, page, _ = pool.shape
    codes = torch.empty(pool.shape, dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty((L, P, Hkv, 2, page // BLOCK), device="cuda")
    for l in range(L):
        x = pool[l].float().view(P, Hkv, 2, page // BLOCK, BLOCK, D)
        scales[l] = _scale_of(torch.nan_to_num(x).abs().amax((-1, -2)))
        codes[l] = (x / scales[l][..., None, None]).to(torch.float8_e4m3fn).view(P, Hkv, 2, page, D)
    return codes, scales


def _rows(c, seed, which):
    """Rows [tokens][layers][kv_heads][D]: a step's as [batch][layers][kv_heads][D], a prompt's as they go
    into a cache, [layers][kv_heads][tokens][D]."""
    T = sum(n for _, n in _spans(c))
    lead = (T, c["layers"], c["kv_heads"], D)
    x = torch.empty(lead if c["step"] else (lead[1], lead[2], T, D), dtype=TYPES[c["type"]], device="cuda")
    if not c["step"]:
        x = x.permute(2, 0, 1, 3)
    if c["op"] == "write":
        x.normal_(generator=_gen(seed, 10 + which))
        if which == 0:
            x *= _channels(seed).to(x.dtype)
    return x


def _places(c):
    """Where a plain program finds the tokens of a write or a read, on the device: sequence, position; of
    the blocks of a write: sequence, number in it, slots held before; each token's block and slot."""
    spans = _spans(c)
    b = np.concatenate([np.full(n, i) for i, (_, n) in enumerate(spans)] or [np.zeros(0)]).astype(np.int64)
    pos = np.concatenate([np.arange(a, a + n) for a, n in spans] or [np.zeros(0)]).astype(np.int64)
    key = b * (1 << 32) + pos // BLOCK
    blocks, of = np.unique(key, return_inverse=True)
    first = np.zeros(len(blocks), np.int64) + BLOCK
    np.minimum.at(first, of, pos % BLOCK)
    to = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    return {"b": to(b), "pos": to(pos), "block_b": to(blocks >> 32), "block_at": to(blocks & 0xffffffff), "held": to(first),
            "of": to(of.reshape(-1)), "slot": to(pos % BLOCK)}


def prepare(case, seed):
    c = dict(DEFAULTS, **case)
    s = {"case": c, "tokens": np.array(_lengths(c), np.int32)}
    s["table"], P = _table(c, seed)
    shape = (c["layers"], P, c["kv_heads"], 2, c["page"], D)
    if c["op"] != "attend":
        # what other tokens of the pages hold: the steps before it
        s["pool"] = (torch.randn(shape, generator=_gen(seed, 4), device="cuda", dtype=torch.bfloat16) * 60).clamp(-MOST, MOST).to(torch.float8_e4m3fn)
        s["scales"] = _power(torch.randint(-8, -5, shape[:4] + (c["page"] // BLOCK,), generator=_gen(seed, 5), device="cuda"))
        s["k"], s["v"] = _rows(c, seed, 0), _rows(c, seed, 1)
        s["first"], s["count"] = (np.array([x[i] for x in _spans(c)], np.int32) for i in (0, 1))
        s["places"] = _places(c)
        return s
    pool = _pool(c, seed, s["table"], P)
    s["pool"], s["scales"] = _quantised(pool) if c["type"] == "e4m3" else (pool, None)
    s["tokens_dev"] = torch.from_numpy(s["tokens"]).cuda().long()
    q = torch.randn((c["batch"], c["layers"], c["q_heads"], D), generator=_gen(seed, 6), device="cuda", dtype=torch.bfloat16)
    q[..., :HOT_DIMS] += HOT_QUERY
    s["q"] = q * _channels(seed + 1).bfloat16() * 0.5
    s["out"] = torch.empty_like(q)
    s["lse"] = torch.empty(q.shape[:3], device="cuda")
    s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------- plain forms ----
def _plain_write(s):
    c, p, sub = s["case"], s["places"], s["case"]["page"] // BLOCK
    codes = s["pool"].view(torch.uint8)
    phys, part = s["table"][p["block_b"], p["block_at"] // sub].long(), p["block_at"] % sub
    old, old_slot = (torch.arange(BLOCK, device="cuda") < p["held"][:, None]).nonzero(as_tuple=True)
    of, slot = p["of"], p["slot"]

    def rows(x, which):
        x = x.float()                                                                 # [tokens][L][Hkv][D]
        full = torch.zeros((phys.numel(), BLOCK) + x.shape[1:], device="cuda")
        full[of, slot] = x
        new, before = _scale_of(full.abs().amax((1, -1))), s["scales"][:, phys, :, which, part]   # [blocks][L][Hkv]
        scale = torch.where(p["held"].view(-1, 1, 1) > 0, torch.maximum(before, new), new)
        s["scales"][:, phys, :, which, part] = scale
        held = codes[:, phys[old], :, which, part[old] * BLOCK + old_slot].view(torch.float8_e4m3fn).float()
        held = (held * (before / scale)[old][..., None]).to(torch.float8_e4m3fn)
        codes[:, phys[old], :, which, part[old] * BLOCK + old_slot] = held.view(torch.uint8)
        x = (x / scale[of][..., None]).to(torch.float8_e4m3fn)
        codes[:, phys[of], :, which, part[of] * BLOCK + slot] = x.view(torch.uint8)

    rows(s["k"], 0)
    rows(s["v"], 1)
    return {"pool": s["pool"], "scales": s["scales"]}


def _plain_read(s):
    c, p = s["case"], s["places"]
    phys, slot = s["table"][p["b"], p["pos"] // c["page"]].long(), p["pos"] % c["page"]
    layer = torch.arange(c["layers"], device="cuda").view(-1, 1)
    head = torch.arange(c["kv_heads"], device="cuda")
    phys, slot = phys.view(-1, 1, 1), slot.view(-1, 1, 1)

    def rows(out, which):
        x = s["pool"].view(torch.uint8)[layer, phys, head, which, slot].view(torch.float8_e4m3fn).float()
        out.copy_(x * s["scales"][layer, phys, head, which, slot // BLOCK][..., None])

    rows(s["k"], 0)
    rows(s["v"], 1)
    return {"k": s["k"], "v": s["v"]}


def _plain_attend(s):
    c = s["case"]
    B, L, Hkv, page = c["batch"], c["layers"], c["kv_heads"], c["page"]
    n = s["tokens_dev"]
    w0 = (n - c["window"]).clamp(min=0) if c["window"] >= 0 else torch.zeros_like(n)
    sinks = w0.clamp(max=c["sinks"])
    most = max([sum((a, x - w)) for x in _lengths(c) for a, w in (_shown(c, x),)] + [1])
    j = torch.arange(most, device="cuda")
    tok = torch.where(j < sinks[:, None], j, j - sinks[:, None] + w0[:, None])        # [B][most]
    held = tok < n[:, None]
    tok = torch.where(held, tok, 0)
    phys = torch.gather(s["table"].long(), 1, tok // page).view(B, 1, 1, -1)
    slot = (tok % page).view(B, 1, 1, -1)
    layer = torch.arange(L, device="cuda").view(-1, 1, 1)
    head = torch.arange(Hkv, device="cuda").view(-1, 1)
    held = held.view(B, 1, 1, -1)

    def rows(which):                                                                  # [B][L][Hkv][most][D]
        if c["type"] == "bf16":
            return torch.where(held[..., None], s["pool"][layer, phys, head, which, slot], 0).float()
        x = s["pool"].view(torch.uint8)[layer, phys, head, which, slot]
        x = torch.where(held[..., None], x, 0).view(torch.float8_e4m3fn).float()
        return x * s["scales"][layer, phys, head, which, slot // BLOCK][..., None]

    q = s["q"].float().view(B, L, Hkv, -1, D)
    x = torch.matmul(q, rows(0).transpose(-1, -2)) * (1.0 / math.sqrt(D))
    x = torch.where(held[..., None, :], x, -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    p = torch.where(z > 0, e / z, 0.0)
    lse = torch.where(z > 0, m + torch.log(z), -math.inf)
    return {"out": torch.matmul(p, rows(1)).view(B, L, -1, D).bfloat16(), "lse": lse.view(B, L, -1)}


# --------------------------------------------------------------- the library ----
def _own(s):
    import paper_2607_10582_gb300 as md
    c, op = s["case"], s["case"]["op"]
    if op == "write":
        md.md_write_cache8(s["k"], s["v"], s["pool"], s["scales"], s["table"], s["first"], s["count"])
        return {"pool": s["pool"], "scales": s["scales"]}
    if op == "read":
        md.md_read_cache8(s["k"], s["v"], s["pool"], s["scales"], s["table"], s["first"], s["count"])
        return {"k": s["k"], "v": s["v"]}
    md.md_attend_cache(s["q"], s["pool"], s["table"], s["tokens"], s["out"], scales=s["scales"],
                       window=c["window"] if c["window"] >= 0 else None, sinks=c["sinks"], lse=s["lse"],
                       workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[state["case"]["op"]](state)


# ------------------------------------------------------------------- exact ----
def _power64(e):
    """2^e in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(y):
    """The e4m3 value nearest to y (ties to even), |y| <= 448, in 64 bits."""
    step = _power64(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return torch.round(y / step) * step


def _exact_write(c, s):
    """Block by block: the largest value decides the scale."""
    pool, scales = s["pool"].double(), s["scales"].double()
    token = 0
    for b, (a, n) in enumerate(_spans(c)):
        x = torch.stack([s["k"][token:token + n], s["v"][token:token + n]], 3).double()      # [n][L][Hkv][2][D]
        token += n
        for i in range(a // BLOCK, -(-(a + n) // BLOCK) if n else 0):
            lo, hi = max(a, i * BLOCK), min(a + n, (i + 1) * BLOCK)
            page, part = int(s["table"][b, i * BLOCK // c["page"]]), i * BLOCK % c["page"] // BLOCK
            new = x[lo - a:hi - a].permute(1, 2, 3, 0, 4)                                    # [L][Hkv][2][m][D]
            part_of, e = torch.frexp(new.abs().amax((-1, -2)).clamp(min=1e-300) / MOST)      # in [1/2, 1)
            scale, held = _power64((e - (part_of == 0.5).int()).clamp(min=-126)), lo - i * BLOCK
            if held:
                was = scales[:, page, :, :, part]
                scale = torch.maximum(scale, was)
                old = pool[:, page, :, :, part * BLOCK:part * BLOCK + held]
                pool[:, page, :, :, part * BLOCK:part * BLOCK + held] = _nearest(old * (was / scale)[..., None, None])
            scales[:, page, :, :, part] = scale
            at = part * BLOCK + held
            pool[:, page, :, :, at:at + hi - lo] = _nearest(new / scale[..., None, None])
    return {"pool": pool, "scales": scales}


def exact(case, seed):
    """From the definitions, sequence by sequence and in 64 bits."""
    c = dict(DEFAULTS, **case)
    if c["op"] == "write" and _blocks(c) > 12000:
        return None
    s = prepare(c, seed)
    if c["op"] == "write":
        return _exact_write(c, s)
    page, L, Hkv, G, n = c["page"], c["layers"], c["kv_heads"], c["q_heads"] // c["kv_heads"], _lengths(c)
    if c["op"] == "read":
        x = torch.zeros((2, sum(n)) + (L, Hkv, D), dtype=torch.float64, device="cuda")
        at = 0
        for b in range(c["batch"]):
            for i in range(0, n[b], page):
                m, phys = min(page, n[b] - i), int(s["table"][b, i // page])
                v = s["pool"][:, phys].double() * s["scales"][:, phys].double().repeat_interleave(BLOCK, -1)[..., None]
                x[:, at:at + m] = v[..., :m, :].permute(2, 3, 0, 1, 4)                       # from [L][Hkv][2][m][D]
                at += m
        return {"k": x[0], "v": x[1]}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        first, w0 = _shown(c, n[b])
        pages = sorted(set(range(-(-first // page))) | set(range(w0 // page, -(-n[b] // page))))
        if not pages:
            continue
        tok = (torch.tensor(pages, device="cuda")[:, None] * page + torch.arange(page, device="cuda")).flatten()
        gone = (tok >= n[b]) | ((tok >= first) & (tok < w0))
        phys = s["table"][b, torch.tensor(pages, device="cuda")].long()
        for l in range(L):
            kv = s["pool"][l].view(torch.uint8)[phys].view(s["pool"].dtype).double()         # [m][Hkv][2][page][D]
            if s["scales"] is not None:
                kv = kv * s["scales"][l, phys].double().repeat_interleave(BLOCK, -1)[..., None]
            k, v = (kv[:, :, i].transpose(0, 1).flatten(1, 2).masked_fill(gone[:, None], 0) for i in (0, 1))
            x = torch.einsum("hgd,hnd->hgn", s["q"][b, l].double().view(Hkv, G, D), k) / math.sqrt(D)
            x = x.masked_fill(gone, -math.inf)
            out[b, l] = torch.einsum("hgn,hnd->hgd", torch.softmax(x, -1), v).flatten(0, 1)
            lse[b, l] = torch.logsumexp(x, -1).flatten()
    return {"out": out, "lse": lse}
