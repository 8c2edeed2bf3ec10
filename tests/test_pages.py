"""The page calls (bounds, scores, selection, attention over selected pages) against plain
64-bit implementations, and their refusals.

Tolerances, from the arithmetic:
  bounds  none: they are stored values.
  scores  a sum of 256 exact products over 16 chained matrix instructions; each may round its
          17 addends and result at 2^-24 of the largest, so 16 * 18 * 2^-24 of the sum of
          the products' sizes bounds it.
  mass    relative: twice the error of a logit (8 chained instructions, as above; numerator and
          sum), and 2^-18 for exp2, the sums and the division.
  out     that, times sum_i p_i |v_i|, with 2^-15 for the weights' two bf16 terms, and the
          output's rounding to bf16 (2^-8 of the value)."""
import math

import numpy as np
import pytest

import paper_2607_10582_gb300 as md
from paper_2607_10582_gb300 import build as mdbuild

torch = pytest.importorskip("torch")
D = 128
mdbuild.build()
gpu = pytest.mark.gpu
CHAIN = 18 * 2.0 ** -24          # of one matrix instruction


def _need_gpu():
    if not torch.cuda.is_available():  # pragma: no cover
        pytest.skip("needs a CUDA GPU")


class Case:
    """A cache whose pages lie anywhere in its pool, NaN wherever no token is."""

    def __init__(self, L, Hq, Hkv, ps, lengths, seed=0, spare=3, width=None, scale=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.L, self.Hq, self.Hkv, self.ps, self.G, self.B = L, Hq, Hkv, ps, Hq // Hkv, len(lengths)
        self.n = np.array(lengths, np.int32)
        self.pages = [-(-x // ps) for x in lengths]
        self.P, self.W = sum(self.pages) + spare, width or max(self.pages) + 2
        ids = np.random.default_rng(seed).permutation(self.P)
        self.table = np.full((self.B, self.W), -1, np.int32)
        self.pool = torch.full((L, self.P, Hkv, 2, ps, D), math.nan, dtype=torch.bfloat16, device="cuda")
        at = 0
        for b, (x, p) in enumerate(zip(lengths, self.pages)):
            self.table[b, :p] = ids[at:at + p]
            at += p
            for i in range(p):
                m = min(ps, x - i * ps)
                self.pool[:, self.table[b, i], :, :, :m] = torch.randn((L, Hkv, 2, m, D), generator=g,
                                                                      device="cuda").bfloat16()
        self.pool[:, :, :, 0] *= scale
        self.q = torch.randn((self.B, L, Hq, D), generator=g, device="cuda").bfloat16()
        self.bt = torch.from_numpy(self.table).cuda()

    def kv(self, b, l, h, pages):
        """float64 K and V of the tokens of these pages, and their (list entry, slot)."""
        k, v, where = [], [], []
        for e, p in enumerate(pages):
            if 0 <= p < self.pages[b] and 0 <= self.table[b, p] < self.P:
                m = min(self.ps, int(self.n[b]) - p * self.ps)
                x = self.pool[l, self.table[b, p], h, :, :m].double()
                k.append(x[0])
                v.append(x[1])
                where += [(e, i) for i in range(m)]
        if not k:
            return None
        return torch.cat(k), torch.cat(v), where

    def bounds(self):
        out = torch.zeros((self.L, self.P, self.Hkv, 2, D), dtype=torch.bfloat16, device="cuda")
        md.md_page_bounds(self.pool, self.bt, self.n, out)
        return out

    def check_attend(self, ids, out, mass):
        top = ids.shape[-1]
        for b in range(self.B):
            for l in range(self.L):
                for h in range(self.Hkv):
                    got = out[b, l, h * self.G:(h + 1) * self.G].double()
                    m = mass[b, l, h].double().view(top, self.ps)
                    kv = self.kv(b, l, h, ids[b, l, h].tolist())
                    if kv is None:
                        assert not got.any() and not m.any()
                        continue
                    k, v, where = kv
                    q = self.q[b, l, h * self.G:(h + 1) * self.G].double()
                    p = torch.softmax(q @ k.T / math.sqrt(D), -1)
                    delta = 8 * CHAIN * float((q.abs() @ k.abs().T).max()) / math.sqrt(D)
                    ref = p @ v
                    tol = 2.0 ** -8 * ref.abs() + (2 * delta + 2.0 ** -15) * (p @ v.abs()) + 1e-30
                    assert ((got - ref).abs() <= tol).all(), (b, l, h, float(((got - ref).abs() / tol).max()))
                    want = torch.zeros_like(m)
                    e, i = torch.tensor(where, device="cuda").T
                    want[e, i] = p.sum(0)
                    assert ((m - want).abs() <= (2 * delta + 2.0 ** -18) * want + 1e-30).all(), (b, l, h)

    def attend(self, ids, **kw):
        out = torch.full_like(self.q, math.nan)
        mass = torch.full((self.B, self.L, self.Hkv, ids.shape[-1] * self.ps), math.nan, device="cuda")
        md.md_attend_pages(self.q, self.pool, self.bt, self.n, ids, out, mass=mass, **kw)
        return out, mass


SHAPES = [
    (1, 1, 1, 16, [1]),
    (1, 12, 2, 16, [448]),
    (2, 16, 2, 32, [33, 0, 31, 32, 700]),
    (3, 8, 1, 16, [1, 15, 16, 17, 0, 300]),
    (1, 6, 2, 32, [5000, 64]),
    (2, 32, 8, 16, [257, 1000]),
    (1, 5, 1, 32, [0, 0]),
    (1, 28, 4, 16, [130 * i for i in range(1, 20)]),
]


@gpu
@pytest.mark.parametrize("L,Hq,Hkv,ps,lengths", SHAPES)
def test_bounds_are_the_keys_extremes(L, Hq, Hkv, ps, lengths):
    _need_gpu()
    c = Case(L, Hq, Hkv, ps, lengths, seed=1)
    first = np.array([p // 2 for p in c.pages], np.int32)
    for f in (None, first):
        got = torch.full((L, c.P, Hkv, 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
        want = got.clone()
        md.md_page_bounds(c.pool, c.bt, c.n, got, first_pages=f)
        for b, x in enumerate(lengths):
            for p in range(0 if f is None else f[b], c.pages[b]):
                k = c.pool[:, c.table[b, p], :, 0, :min(ps, x - p * ps)]
                want[:, c.table[b, p], :, 0], want[:, c.table[b, p], :, 1] = k.amin(-2), k.amax(-2)
        assert torch.equal(got, want)


@gpu
@pytest.mark.parametrize("L,Hq,Hkv,ps,lengths", SHAPES)
def test_scores_bound_the_logits(L, Hq, Hkv, ps, lengths):
    _need_gpu()
    c = Case(L, Hq, Hkv, ps, lengths, seed=2)
    bounds = c.bounds()
    got = torch.full((c.B, L, Hkv, c.W), 7.0, device="cuda")
    md.md_page_scores(c.q, bounds, c.bt, c.n, got, page_size=ps)
    for b in range(c.B):
        for l in range(L):
            for h in range(Hkv):
                assert (got[b, l, h, c.pages[b]:] == 7.0).all()
                if not c.pages[b]:
                    continue
                x = bounds[l, torch.from_numpy(c.table[b, :c.pages[b]]).cuda().long(), h].double()
                q = c.q[b, l, h * c.G:(h + 1) * c.G].double()
                ref = (q.clamp(min=0) @ x[:, 1].T + q.clamp(max=0) @ x[:, 0].T).amax(0) / math.sqrt(D)
                size = (q.abs() @ x.abs().amax(1).T).amax(0) / math.sqrt(D)
                s = got[b, l, h, :c.pages[b]].double()
                assert ((s - ref).abs() <= 16 * CHAIN * size).all()
                k, _, where = c.kv(b, l, h, range(c.pages[b]))
                page = torch.tensor([e for e, _ in where], device="cuda")
                logit = (q @ k.T).amax(0) / math.sqrt(D)
                assert (logit <= s[page] + 16 * CHAIN * size[page]).all()


def _top_ref(x, n, top, first, last):
    """Rows of scores -> page lists, by sorting (score, index)."""
    if n <= top:
        return list(range(n)) + [-1] * (top - n)
    mid = list(range(first, n - last))
    key = [(-math.inf if math.isnan(x[i]) else -x[i] if x[i] != math.inf else -1e300, i) for i in mid]
    keep = sorted(i for _, i in sorted(key)[:top - first - last])
    return list(range(first)) + keep + list(range(n - last, n))


@gpu
@pytest.mark.parametrize("pages,top,first,last", [
    ([1, 0, 5, 4], 4, 1, 1), ([17, 16, 15], 16, 0, 0), ([100, 99, 3], 2, 1, 1), ([700, 513, 512], 40, 3, 5),
    ([1025, 64, 2], 1000, 0, 1), ([4097], 64, 1, 1), ([16384, 9000, 40], 300, 1, 2), ([5000], 1, 0, 0),
    ([5000, 20], 1, 1, 0), ([300], 299, 100, 100),
])
@pytest.mark.parametrize("kind", ["normal", "ties", "special"])
def test_selection_takes_the_highest_and_the_first_of_equals(pages, top, first, last, kind):
    _need_gpu()
    rng = np.random.default_rng(len(pages) * top)
    B, L, Hkv, W = len(pages), 2, 2, max(pages)
    x = rng.standard_normal((B, L, Hkv, W)).astype(np.float32)
    if kind == "ties":
        x = np.round(x)
        x[x == 0] = np.where(rng.random((x == 0).sum()) < 0.5, -0.0, 0.0)
    elif kind == "special":
        x[rng.random(x.shape) < 0.05] = np.nan
        x[rng.random(x.shape) < 0.05] = np.inf
        x[rng.random(x.shape) < 0.3] = -np.inf
        x[rng.random(x.shape) < 0.05] = 1e-42
    for b, p in enumerate(pages):
        x[b, :, :, p:] = np.nan                       # not the sequence's pages
        if p > top:
            x[b, :, :, :first] = np.nan               # not read
    ids = torch.full((B, L, Hkv, top), 12345, dtype=torch.int32, device="cuda")
    md.md_page_top(torch.from_numpy(x).cuda(), np.array(pages, np.int32) * 16, ids, page_size=16, first=first, last=last)
    got = ids.cpu().numpy()
    for b, p in enumerate(pages):
        for l in range(L):
            for h in range(Hkv):
                assert got[b, l, h].tolist() == _top_ref(x[b, l, h].tolist(), p, top, first, last), (b, l, h)


def _pick(c, top, seed, holes=False):
    rng = np.random.default_rng(seed)
    ids = np.full((c.B, c.L, c.Hkv, top), -1, np.int32)
    for b in range(c.B):
        for l in range(c.L):
            for h in range(c.Hkv):
                some = np.sort(rng.permutation(c.pages[b])[:top])
                if holes and len(some):
                    some = np.where(rng.random(len(some)) < 0.4, rng.choice([-1, -7, c.pages[b], 1 << 30], len(some)), some)
                ids[b, l, h, :len(some)] = some
    return torch.from_numpy(ids).cuda()


@gpu
@pytest.mark.parametrize("top", [1, 2, 9, 40, 333])
@pytest.mark.parametrize("L,Hq,Hkv,ps,lengths", SHAPES)
def test_attention_over_listed_pages(L, Hq, Hkv, ps, lengths, top):
    _need_gpu()
    c = Case(L, Hq, Hkv, ps, lengths, seed=3)
    ids = _pick(c, top, 4)
    out, mass = c.attend(ids)
    c.check_attend(ids, out, mass)
    again = torch.full_like(out, math.nan)
    md.md_attend_pages(c.q, c.pool, c.bt, c.n, ids, again)         # without the masses
    assert torch.equal(again, out)


@gpu
@pytest.mark.parametrize("ps,lengths,top", [(16, [3000, 1, 0, 170], 60), (32, [3000, 200], 94)])
def test_lists_with_holes_and_tables_with_strangers(ps, lengths, top):
    """Entries that are no page of the sequence, and table entries outside the pool, count
    as pages without tokens."""
    _need_gpu()
    c = Case(2, 12, 2, ps, lengths, seed=5)
    c.table[0, 5], c.table[0, 90], c.table[0, 50] = -1, c.P, 1 << 30
    c.bt = torch.from_numpy(c.table).cuda()
    ids = _pick(c, top, 6, holes=True)
    ids[0, 1, 1] = -1                                              # a row of nothing
    out, mass = c.attend(ids)
    c.check_attend(ids, out, mass)


@gpu
def test_pages_outside_the_pool_are_selected_last():
    """A table entry outside the pool is a page without tokens: no page of scores below 0 gives
    way to it, whatever the queries."""
    _need_gpu()
    c = Case(2, 16, 2, 16, [500, 333], seed=23)
    c.pool[:, :, :, 0] = -(c.pool[:, :, :, 0].abs())
    c.q = c.q.abs()
    c.q[1, 0, 0, 0] = math.inf
    bounds = c.bounds()
    for b, pg, entry in ((0, 4, c.P), (0, 18, -1), (1, 1, 1 << 30), (1, 16, -(1 << 31))):
        c.table[b, pg] = entry
    c.bt = torch.from_numpy(c.table).cuda()
    scores = torch.zeros((2, 2, 2, c.W), device="cuda")
    md.md_page_scores(c.q, bounds, c.bt, c.n, scores, page_size=16)
    assert (scores[0][..., [4, 18]] == -math.inf).all() and (scores[1][..., [1, 16]] == -math.inf).all()
    assert (scores[0, :, :, [0, 1, 2, 3, 5, 31]] < 0).all() and (scores[0, :, :, 5] > -math.inf).all()
    ids = torch.zeros((2, 2, 2, 19), dtype=torch.int32, device="cuda")
    md.md_page_top(scores, c.n, ids, page_size=16, first=0, last=0)
    assert not (ids[0] == 4).any() and not (ids[0] == 18).any() and not (ids[1] == 1).any() and not (ids[1] == 16).any()


@gpu
@pytest.mark.parametrize("scale", [0.0, 30.0, 300.0])
def test_flat_and_steep_softmax(scale):
    """Equal logits, and logits of hundreds, where the weights round to one token."""
    _need_gpu()
    c = Case(1, 16, 2, 16, [900, 37], seed=7, scale=scale)
    ids = _pick(c, 57, 8)
    out, mass = c.attend(ids)
    c.check_attend(ids, out, mass)


@gpu
@pytest.mark.parametrize("lengths,top", [([16], 1), ([700, 3000], 188), ([3000] * 40, 60)])
@pytest.mark.parametrize("low,high", [(-10.0, -10.0), (-60.0, -9.0), (-60.0, 60.0), (40.0, -40.0)])
def test_logits_far_from_zero(lengths, top, low, high):
    """All logits of a list, or of its parts, at +-100 to +-680: the weights' base moves as far."""
    _need_gpu()
    c = Case(2, 16, 2, 16, lengths, seed=11)
    g = torch.Generator(device="cuda").manual_seed(12)
    s = torch.where(torch.rand(D, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    c.q = (s * (1 + 0.02 * torch.randn((c.B, c.L, c.Hq, D), generator=g, device="cuda"))).bfloat16()
    level = torch.where(torch.rand(c.P, generator=g, device="cuda") < 0.5, low, high)[:, None, None, None]
    noise = 0.05 * torch.randn((c.L, c.P, c.Hkv, c.ps, D), generator=g, device="cuda")
    k = c.pool[:, :, :, 0]
    c.pool[:, :, :, 0] = torch.where(k.isnan(), k, (s * level + noise).bfloat16())
    ids = _pick(c, top, 13)
    c.check_attend(ids, *c.attend(ids))


@gpu
def test_infinite_and_nan_tokens_stay_in_their_heads():
    _need_gpu()
    c = Case(1, 4, 2, 16, [200, 100], seed=9)
    page = int(c.table[0, 3])
    c.pool[0, page, 1, 0, 4, 7] = math.nan                          # a key of KV head 1
    ids = _pick(c, 13, 10)
    out, mass = c.attend(ids)
    assert out[0, 0, 2:].isnan().all() and not out[0, 0, :2].isnan().any() and not out[1].isnan().any()
    bounds = c.bounds()
    assert bounds[0, page, 1, :, 7].isnan().all() and not bounds[0, page, 1, :, 8].isnan().any()
    scores = torch.zeros((2, 1, 2, c.W), device="cuda")
    md.md_page_scores(c.q, bounds, c.bt, c.n, scores, page_size=16)
    assert scores[0, 0, 1, 3].isnan() and scores.isnan().sum() == 1
    few = torch.empty((2, 1, 2, 3), dtype=torch.int32, device="cuda")
    md.md_page_top(scores, c.n, few, page_size=16, first=1, last=1)
    assert few[0, 0, 1].tolist() == [0, 3, 12]                      # the page that holds it is attended


@gpu
@pytest.mark.parametrize("value", [math.inf, -math.inf])
@pytest.mark.parametrize("ps,lengths,top", [(16, [200], 13), (32, [3000] * 40, 60), (16, [700, 3001], 188), (16, [7], 1)])
def test_infinite_values_stay_infinite(ps, lengths, top, value):
    """An infinite value makes its channel infinite in the heads that attend it, as in the
    formula: in a full tile, and in the last token of a partly filled one."""
    _need_gpu()
    c = Case(2, 16, 2, ps, lengths, seed=21)
    b, n = len(lengths) - 1, lengths[-1]
    for tok, ch in ((n - 1, 5), (min(n - 1, 3 * ps + 2), 77)):
        c.pool[0, c.table[b, tok // ps], 1, 1, tok % ps, ch] = value
    ids = torch.full((c.B, 2, 2, top), -1, dtype=torch.int32)
    for i in range(c.B):
        keep = sorted(({3, c.pages[i] - 1} | set(range(min(top - 2, c.pages[i])))) & set(range(c.pages[i])))
        ids[i, :, :, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
    out, mass = c.attend(ids.cuda())
    want = torch.zeros_like(out, dtype=torch.bool)
    want[b, 0, 8:, 5] = want[b, 0, 8:, 77] = True
    assert torch.equal(out == value, want) and not out.isnan().any() and not mass.isnan().any()


@gpu
@pytest.mark.parametrize("lengths,top", [([900], 57), ([900] * 40, 57)])
def test_infinite_values_of_any_weight_and_sign(lengths, top):
    """A weight far below what 32 bits hold is above 0 all the same; values of both signs, or
    a NaN, make their channel NaN; tokens that are not listed are not looked at."""
    _need_gpu()
    c = Case(1, 16, 2, 16, lengths, seed=22, scale=300.0)
    clean = c.pool.clone()
    at = [c.table[0, i // 16] for i in range(900)]
    for tok, ch, x in ((40, 3, math.inf), (300, 3, math.inf), (500, 60, -math.inf), (17, 90, math.inf), (899, 90, -math.inf),
                       (700, 127, math.nan), (701, 126, math.inf), (320, 30, math.inf)):
        c.pool[0, at[tok], 0, 1, tok % 16, ch] = x
    ids = torch.arange(top, dtype=torch.int32, device="cuda").repeat(c.B, 1, 2, 1)
    ids[..., 20] = -1                                   # the page of token 320
    out, mass = c.attend(ids)
    c.pool = clean
    want, same = c.attend(ids)
    want[0, 0, :8, 3], want[0, 0, :8, 60], want[0, 0, :8, 126] = math.inf, -math.inf, math.inf
    for ch in (90, 127):
        assert out[0, 0, :8, ch].isnan().all()
        out[0, 0, :8, ch] = want[0, 0, :8, ch] = 0.0
    assert torch.equal(out, want) and torch.equal(mass, same)


@gpu
def test_results_repeat_and_streams_are_kept():
    _need_gpu()
    c = Case(2, 16, 2, 32, [9000, 40, 2500], seed=11)
    ids = _pick(c, 70, 12)
    out, mass = c.attend(ids)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        late = torch.full_like(ids, -1)
        for _ in range(20):
            late.copy_(ids)
        for _ in range(5):
            o, m = c.attend(late)
        s.synchronize()
    assert torch.equal(o, out) and torch.equal(m, mass)


@gpu
def test_launches_on_several_streams_at_once():
    """Rows of one CTA each, with masses and without, in flight together."""
    _need_gpu()
    c = Case(4, 16, 2, 16, [3000] * 40, seed=14)
    ids = _pick(c, 188, 15)
    out, mass = c.attend(ids)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    torch.cuda.synchronize()
    for i in range(12):
        o = torch.empty_like(out)
        m = torch.empty_like(mass) if i % 4 else None
        got.append((o, m))
        md.md_attend_pages(c.q, c.pool, c.bt, c.n, ids, o, mass=m, stream=streams[i % 3])
    torch.cuda.synchronize()
    for o, m in got:
        assert torch.equal(o, out) and (m is None or torch.equal(m, mass))


@gpu
def test_calls_without_the_c_module_are_the_same(monkeypatch):
    _need_gpu()
    c = Case(2, 16, 2, 16, [700, 40, 0], seed=15)
    got = []
    for b in (md._binding(), md._NoCalls):
        monkeypatch.setattr(md, "_torch_calls", None)
        monkeypatch.setattr(md, "_fast", b)
        bounds, scores = c.bounds(), torch.zeros((3, 2, 2, c.W), device="cuda")
        ids = torch.zeros((3, 2, 2, 9), dtype=torch.int32, device="cuda")
        md.md_page_scores(c.q, bounds, c.bt, c.n, scores, page_size=16)
        md.md_page_top(scores, c.n.tolist(), ids, page_size=16, first=2, last=3)
        got.append((bounds, scores, ids) + c.attend(ids))
    assert all(torch.equal(x, y) for x, y in zip(*got)) and got[0][3].any()


@gpu
def test_pages_past_32_bit_offsets():
    """A pool of more than 2^32 bytes and 2^31 elements: pages at its end."""
    _need_gpu()
    L, Hkv, ps, P = 2, 1, 32, 300000
    pool = torch.empty((L, P, Hkv, 2, ps, D), dtype=torch.bfloat16, device="cuda")
    c = Case(L, 8, Hkv, ps, [200], seed=13)
    table = np.arange(P - 1, P - 1 - c.W, -1).astype(np.int32)[None]
    at = torch.from_numpy(table[0, :c.pages[0]].copy()).cuda().long()
    pool[:, at] = c.pool[:, torch.from_numpy(c.table[0, :c.pages[0]]).cuda().long()]
    c.pool, c.table, c.P, c.bt = pool, table, P, torch.from_numpy(table).cuda()
    ids = _pick(c, 7, 14)
    out, mass = c.attend(ids)
    c.check_attend(ids, out, mass)
    bounds = c.bounds()
    k = pool[:, at[:6], :, 0]
    assert torch.equal(bounds[:, at[:6], :, 0], k.amin(-2)) and torch.equal(bounds[:, at[:6], :, 1], k.amax(-2))


# ---------------------------------------------------------------- refusals ----
A = 1 << 20      # an address that nothing reads: a call that is not refused would need a GPU
N = np.array([100, 0], np.int32)
COMMON = dict(batch=2, L=2, Hkv=2, ps=16, P_max=8, P=64)


def _geometry(**kw):
    bad = [dict(batch=0), dict(batch=257), dict(L=0), dict(L=256), dict(Hkv=0), dict(ps=8), dict(P_max=0), dict(P=0),
           dict(P_max=6), dict(P_max=1 << 20), dict(P=1 << 30)]
    return [dict(COMMON, **b) for b in bad] + [dict(COMMON, **kw)] * bool(kw)


def test_refusals_of_geometry():
    lib, bad = md.lib(), md.MD_ERR_INVALID_ARG
    n = N.ctypes.data
    for c in _geometry():
        g = (c["L"], c["Hkv"], c["ps"], c["P_max"], c["P"])
        h = (c["L"], 16, c["Hkv"], c["ps"], c["P_max"], c["P"])
        assert lib.md_page_bounds(A, A, n, None, A, c["batch"], *g, None) == bad, c
        assert lib.md_page_scores(A, A, A, n, A, c["batch"], *h, None) == bad, c
        assert lib.md_attend_pages(A, A, A, n, A, A, None, c["batch"], *h, 4, None) == bad, c
        if c["P"] == COMMON["P"]:
            assert lib.md_page_top(A, n, A, c["batch"], *g[:4], 4, 1, 1, None) == bad, c
    neg = np.array([-1, 0], np.int32)
    assert lib.md_page_bounds(A, A, neg.ctypes.data, None, A, 2, 2, 2, 16, 8, 64, None) == bad
    assert lib.md_page_bounds(A, A, n, neg.ctypes.data, A, 2, 2, 2, 16, 8, 64, None) == bad


def test_refusals_of_arguments():
    lib, bad, n = md.lib(), md.MD_ERR_INVALID_ARG, N.ctypes.data
    g, h = (2, 2, 2, 16, 8, 64), (2, 2, 16, 2, 16, 8, 64)
    for x in ((None, A, n, None, A), (A + 8, A, n, None, A), (A, None, n, None, A), (A, A, None, None, A),
              (A, A, n, None, None), (A, A, n, None, A + 2)):
        assert lib.md_page_bounds(*x, *g, None) == bad, x
    for x in ((None, A, A, n, A), (A + 8, A, A, n, A), (A, None, A, n, A), (A, A, None, n, A), (A, A, A, None, A),
              (A, A, A, n, None)):
        assert lib.md_page_scores(*x, *h, None) == bad, x
    for x in ((None, A, A, n, A, A), (A, A + 4, A, n, A, A), (A, A, None, n, A, A), (A, A, A, None, A, A),
              (A, A, A, n, None, A), (A, A, A, n, A, None), (A, A, A, n, A, A + 4)):
        assert lib.md_attend_pages(*x, None, *h, 4, None) == bad, x
    for heads in ((17, 2), (1, 2), (18, 2), (0, 2)):
        assert lib.md_page_scores(A, A, A, n, A, 2, 2, *heads, 16, 8, 64, None) == bad, heads
        assert lib.md_attend_pages(A, A, A, n, A, A, None, 2, 2, *heads, 16, 8, 64, 4, None) == bad, heads
    for top in (0, -1, md.MD_MAX_TOP_TOKENS // 16 + 1):
        assert lib.md_attend_pages(A, A, A, n, A, A, None, *h, top, None) == bad, top
    for top, first, last in ((0, 0, 0), (4, -1, 1), (4, 1, -1), (4, 3, 2), (4, 5, 0), (4, 0, 5)):
        assert lib.md_page_top(A, n, A, 2, 2, 2, 16, 8, top, first, last, None) == bad, (top, first, last)
    assert lib.md_page_top(None, n, A, 2, 2, 2, 16, 8, 4, 1, 1, None) == bad
    assert lib.md_page_top(A, n, None, 2, 2, 2, 16, 8, 4, 1, 1, None) == bad


def test_binding_refuses_other_shapes_and_host_tensors():
    pool = torch.zeros((1, 4, 2, 2, 16, D), dtype=torch.bfloat16)
    bounds = torch.zeros((1, 4, 2, 2, D), dtype=torch.bfloat16)
    bt, q = torch.zeros((1, 4), dtype=torch.int32), torch.zeros((1, 1, 8, D), dtype=torch.bfloat16)
    scores, ids = torch.zeros((1, 1, 2, 4)), torch.zeros((1, 1, 2, 2), dtype=torch.int32)
    for call in (lambda: md.md_page_bounds(pool, bt, [10], bounds), lambda: md.md_page_bounds(pool, bt, [], bounds),
                 lambda: md.md_page_scores(q, bounds, bt, [10], scores, page_size=16),
                 lambda: md.md_page_top(scores, [10], ids, page_size=16),
                 lambda: md.md_attend_pages(q, pool, bt, [10], ids, q)):
        with pytest.raises(md.MemDecayError):
            call()
