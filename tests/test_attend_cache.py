"""Attention over a cache that the caller owns (md_attend_cache) against a plain 64-bit
implementation, and its refusals.

Tolerances, from the arithmetic (a matrix instruction rounds its 17 addends and result at 2^-24 of
the largest, 18 x 2^-24 of the sum of the products' sizes; a logit's chain has 8):
  logit   8 x 18 x 2^-24 of sum |q k| / sqrt(128), and for E4M3 the part of a query below 2^-29 of the
          head's largest element, 2^-39 max|q| sum |k|
  out     twice a logit's error, 2^-11 for a weight's rounding (E4M3: f16; BF16: two bf16 terms, less) and 2^-15 for exp2,
          the sums and the division, times sum p |v|; 2^-30 sum |v| for weights in f16's subnormal range
          (at most 2^-25, where the largest weight is 2^5 at least); the output's rounding to bf16, 2^-8
  lse     a logit's error, its roundings (2^-21 of the largest logit), and those of the sum of
          exponentials: 2^-20, and 2^-24 for each of a lane's additions, n / 8 at most"""
import ctypes
import math

import numpy as np
import pytest

import paper_2607_10582_gb300 as md
from paper_2607_10582_gb300 import build as mdbuild
from tests.attend_forms import FORMS

torch = pytest.importorskip("torch")
D = 128
mdbuild.build()
gpu = pytest.mark.gpu
CHAIN = 18 * 2.0 ** -24


def _need_gpu():
    if not torch.cuda.is_available():  # pragma: no cover
        pytest.skip("needs a CUDA GPU")


class Case:
    """A cache whose pages lie anywhere in its pool, NaN wherever no token is (scales too)."""

    def __init__(self, kind, L, Hq, Hkv, ps, lengths, seed=0, spare=3, scale=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.kind, self.L, self.Hq, self.Hkv, self.ps, self.G, self.B = kind, L, Hq, Hkv, ps, Hq // Hkv, len(lengths)
        self.n = np.array(lengths, np.int32)
        self.pages = [-(-x // ps) for x in lengths]
        self.P, self.W = sum(self.pages) + spare, min(max(self.pages) + 2, (1 << 18) // ps)
        ids = np.random.default_rng(seed).permutation(self.P)
        self.table = np.full((self.B, self.W), -1, np.int32)
        shape = (L, self.P, Hkv, 2, ps, D)
        x = torch.randn(shape, generator=g, device="cuda")
        x[:, :, :, 0] *= scale
        self.held = torch.zeros((self.P, ps), dtype=torch.bool, device="cuda")
        at = 0
        for b, (m, p) in enumerate(zip(lengths, self.pages)):
            self.table[b, :p] = ids[at:at + p]
            at += p
            for i in range(p):
                self.held[self.table[b, i], :min(ps, m - i * ps)] = True
        held = self.held[None, :, None, None, :, None]
        if kind == "bf16":
            self.pool, self.scales = torch.where(held, x, math.nan).bfloat16(), None
        else:                                                     # any scales: powers of two far apart
            e = torch.randint(-9, 10, shape[:4] + (ps // 16,), generator=g, device="cuda")
            e[:, :, :, 0] = e[:, :, :, 0] // 5
            s = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
            x = torch.where(held, x.view(shape[:4] + (ps // 16, 16, D)).mul(40).view(shape), math.nan)
            self.pool = x.to(torch.float8_e4m3fn)
            used = self.held.view(self.P, ps // 16, 16).any(-1)[None, :, None, None]
            s[:, :, :, 0] *= 2.0 ** -5
            self.scales = torch.where(used, s, math.nan)
        self.q = torch.randn((self.B, L, Hq, D), generator=g, device="cuda").bfloat16()
        self.bt = torch.from_numpy(self.table).cuda()

    def rows(self, b, l, h, toks):
        phys, slot = torch.from_numpy(self.table[b, toks // self.ps]).cuda().long(), torch.from_numpy(toks % self.ps).cuda()
        x = self.pool[l, phys, h].view(torch.uint8 if self.scales is not None else torch.int16)
        x = x[torch.arange(len(toks), device="cuda"), :, slot].view(self.pool.dtype).double()      # [n][2][D]
        if self.scales is not None:
            x = x * self.scales[l, phys, h, :, slot // 16].double()[..., None]
        return x[:, 0], x[:, 1]

    def visible(self, b, window, sinks):
        i = np.arange(self.n[b])
        i = i[(i < sinks) | (i >= int(self.n[b]) - (1 << 40 if window is None else window))]
        phys = self.table[b, i // self.ps]
        return i[(phys >= 0) & (phys < self.P)]

    def check(self, out, lse, window=None, sinks=0):
        for b in range(self.B):
            toks = self.visible(b, window, sinks)
            for l in range(self.L):
                for h in range(self.Hkv):
                    heads = slice(h * self.G, (h + 1) * self.G)
                    got, z = out[b, l, heads].double(), lse[b, l, heads].double()
                    if not len(toks):
                        assert not got.any() and (z == -math.inf).all(), (b, l, h)
                        continue
                    k, v = self.rows(b, l, h, toks)
                    q = self.q[b, l, heads].double()
                    x = q @ k.T / math.sqrt(D)
                    p = torch.softmax(x, -1)
                    delta = float((8 * CHAIN * (q.abs() @ k.abs().T) +
                                   2.0 ** -39 * q.abs().amax(1, keepdim=True) * k.abs().sum(1)).max()) / math.sqrt(D)
                    ref = p @ v
                    if math.isnan(delta):                         # a visible key is NaN: so is all that it enters
                        assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(z.isnan(), x.isnan().any(1))
                        continue
                    tol = 2.0 ** -8 * ref.abs() + (2 * delta + 2.0 ** -11 + 2.0 ** -15) * (p @ v.abs()) + \
                        2.0 ** -30 * v.abs().sum(0) + 2.0 ** -133
                    assert ((got - ref).abs() <= tol).all(), (b, l, h, float(((got - ref).abs() / tol).max()))
                    want = torch.logsumexp(x, -1)
                    tol = delta + 2.0 ** -21 * float(x.abs().max()) + 2.0 ** -20 + len(toks) / 8 * 2.0 ** -24
                    assert ((z - want).abs() <= tol).all(), (b, l, h, float(((z - want).abs() / tol).max()))

    def attend(self, workspace=False, **kw):
        out = torch.full_like(self.q, math.nan)
        lse = torch.full((self.B, self.L, self.Hq), math.nan, device="cuda")
        ws = torch.full((md.MD_ATTEND_WORKSPACE,), 255, dtype=torch.uint8, device="cuda") if workspace else None
        md.md_attend_cache(self.q, self.pool, self.bt, self.n, out, scales=self.scales, lse=lse, workspace=ws, **kw)
        return out, lse


SHAPES = [
    (1, 1, 1, 16, [1]),
    (1, 12, 2, 16, [448]),
    (2, 16, 2, 32, [33, 0, 31, 32, 700]),
    (3, 8, 1, 16, [1, 15, 16, 17, 0, 300]),
    (1, 6, 2, 32, [5000, 64]),
    (2, 32, 8, 16, [257, 1000]),
    (1, 5, 1, 32, [0, 0]),
    (1, 28, 4, 16, [130 * i for i in range(1, 20)]),
    (1, 7, 1, 16, [20011]),
]
KINDS = ["e4m3", "bf16"]


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("L,Hq,Hkv,ps,lengths", SHAPES)
def test_all_tokens(kind, L, Hq, Hkv, ps, lengths):
    _need_gpu()
    c = Case(kind, L, Hq, Hkv, ps, lengths, seed=3)
    out, lse = c.attend()
    c.check(out, lse)
    again = torch.full_like(out, math.nan)
    md.md_attend_cache(c.q, c.pool, c.bt, c.n, again, scales=c.scales)      # without the logarithms
    assert torch.equal(again, out)
    c.check(*c.attend(workspace=True))


@gpu
@pytest.mark.parametrize("kind,L,Hkv,workspace,lengths,form", FORMS)
def test_every_form(kind, L, Hkv, workspace, lengths, form):
    _need_gpu()
    c = Case(kind, L, 5 * Hkv, Hkv, 16 if form[0] % 3 else 32, lengths, seed=sum(lengths))
    c.check(*c.attend(bool(workspace)))
    window = max(0, max(lengths) - 3)
    c.check(*c.attend(bool(workspace), window=window, sinks=2), window, 2)


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_the_largest_batch(kind):
    """256 ragged sequences, some empty, one long, in the order that the launch sorts them into."""
    _need_gpu()
    c = Case(kind, 1, 8, 2, 16, [(b * 37) % 200 if b != 101 else 6000 for b in range(md.MD_MAX_BATCH)], seed=31)
    for workspace in (False, True):
        c.check(*c.attend(workspace))


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 5), (1, 0), (1, 1), (5, 0), (16, 16), (17, 4), (100, 33), (1000, 16),
                                          (None, 7), (1 << 40, 1 << 40), (3, 4000)])
@pytest.mark.parametrize("L,Hq,Hkv,ps,lengths", [SHAPES[2], SHAPES[3], SHAPES[4]])
def test_windows_and_sinks(kind, L, Hq, Hkv, ps, lengths, window, sinks):
    """Also: tokens that the window hides hold NaN, and pages without visible ones are in no table."""
    _need_gpu()
    c = Case(kind, L, Hq, Hkv, ps, lengths, seed=4)
    shown = torch.zeros_like(c.held)
    for b in range(c.B):
        toks = c.visible(b, window, sinks)
        for pg in range(c.pages[b]):
            some = toks[toks // ps == pg] % ps
            shown[c.table[b, pg], torch.from_numpy(some).cuda()] = True
            if not len(some):
                c.table[b, pg] = (-1, c.P, 1 << 30)[pg % 3]
    raw = c.pool.view(torch.int16 if kind == "bf16" else torch.uint8)
    raw.masked_fill_(~shown[None, :, None, None, :, None], 0x7fc0 if kind == "bf16" else 0xff)
    c.bt = torch.from_numpy(c.table).cuda()
    for workspace in (False, True):
        c.check(*c.attend(workspace, window=window, sinks=sinks), window, sinks)


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_entries_outside_the_pool_are_pages_without_tokens(kind):
    _need_gpu()
    c = Case(kind, 2, 12, 2, 16, [3000, 40, 20], seed=5)
    c.table[0, [5, 90, 50, 51, 52]] = [-1, c.P, 1 << 30, -(1 << 31), -7]
    c.table[2] = -1                                               # nothing of the sequence is there
    c.bt = torch.from_numpy(c.table).cuda()
    for workspace in (False, True):
        c.check(*c.attend(workspace))
        c.check(*c.attend(workspace, window=800, sinks=3), 800, 3)


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scale", [0.0, 30.0, -200.0])
def test_large_and_equal_logits(kind, scale):
    """All logits equal; weights that one token has alone, and maxima that rise far within a row."""
    _need_gpu()
    c = Case(kind, 1, 16, 2, 32, [4000, 129, 1], seed=6, scale=scale)
    for workspace in (False, True):
        c.check(*c.attend(workspace))                             # e4m3: keys beyond 448 scales are NaN
    c = Case(kind, 1, 16, 2, 32, [4000, 129, 1], seed=6)
    (c.pool if kind == "bf16" else c.scales)[:, :, :, 0] *= scale
    if scale > 0:                                                 # rising along the sequence
        for b in range(3):
            for i, pg in enumerate(c.table[b, :c.pages[b]]):
                k = c.pool[:, pg, :, 0].float() * ((i + 1) / c.pages[b])
                c.pool[:, pg, :, 0] = k.to(c.pool.dtype)
    for workspace in (False, True):
        c.check(*c.attend(workspace))


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** 40])
def test_queries_of_any_size(kind, size):
    """Elements of a query far below its largest, zeros, and rows of zeros."""
    _need_gpu()
    c = Case(kind, 1, 8, 2, 16, [500, 3], seed=7)
    c.q = (c.q.float() * 2.0 ** torch.randint(-40, 1, c.q.shape, device="cuda")).bfloat16()
    c.q[0, 0, 3] = 0
    c.q[0, 0, 1, 5:] = 0
    if c.scales is not None:
        c.scales[:, :, :, 0] /= size
    else:
        c.pool[:, :, :, 0] = (c.pool[:, :, :, 0].float() / size).bfloat16()
    c.q = (c.q.float() * size).bfloat16()
    c.check(*c.attend())


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** 100])
def test_values_of_any_size(kind, size):
    """Values near the ends of the range: no sum on the way overflows, none falls to zero."""
    _need_gpu()
    c = Case(kind, 1, 8, 2, 16, [500, 3, 40], seed=17)
    if c.scales is not None:
        c.scales[:, :, :, 1] *= size
    else:
        c.pool[:, :, :, 1] = (c.pool[:, :, :, 1].float() * size).bfloat16()
    for workspace in (False, True):
        out, lse = c.attend(workspace)
        assert out.isfinite().all() and (out != 0).any(-1).all()
        c.check(out, lse)


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_the_largest_values_at_the_largest_weights(kind):
    """131,071 values of 1.75 x 2^99 that all exceed their warp's first maximum by 9.9 in log2, just too
    little to rescale: sums of up to 2^(17 + 9.9 + 99.8), below 2^128 even in one place."""
    _need_gpu()
    n, low = 131071, 8192                                         # each of up to 128 warps sees 32 low ones or more first
    c = Case(kind, 1, 4, 1, 16, [n], seed=18, spare=0)
    phys = c.bt[0, :c.pages[0]].long()
    x = torch.zeros((c.pages[0], 16, D), device="cuda")
    c.q.fill_(1)                                                  # logits 128 k / sqrt(128), x log2(e): 16.32 k
    k, v = (16.0, 448.0) if kind == "e4m3" else (0.605, 1.75 * 2.0 ** 99)
    x[low // 16:] = k
    c.pool[0, phys, 0, 0] = x.to(c.pool.dtype)
    c.pool[0, phys, 0, 1] = torch.full_like(x, v).to(c.pool.dtype)
    c.pool[0, phys[-1], 0, :, 15] = math.nan                      # no token
    if c.scales is not None:
        c.scales[:, :, :, 0], c.scales[:, :, :, 1] = 0.605 / 16, 2.0 ** 91
    for workspace in (False, True):
        out, lse = c.attend(workspace)
        assert out.isfinite().all()
        c.check(out, lse)


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_nan_where_a_visible_token_has_it(kind):
    _need_gpu()
    nan = 0x7fc0 if kind == "bf16" else 0x7f
    raw = torch.int16 if kind == "bf16" else torch.uint8
    c = Case(kind, 1, 16, 2, 16, [300, 90], seed=8)
    c.pool.view(raw)[0, c.table[0, 4], 1, 1, 3, 17] = nan         # a value: its channel of that head group
    c.pool.view(raw)[0, c.table[1, 2], 0, 0, 3, 5] = nan          # a key: all of its group
    for workspace in (False, True):
        out, lse = c.attend(workspace)
        bad = torch.zeros_like(out, dtype=torch.bool)
        bad[0, 0, 8:, 17] = True
        bad[1, 0, :8] = True
        assert torch.equal(out.isnan(), bad)
        assert lse.isnan().nonzero().tolist() == [[1, 0, h] for h in range(8)]
        out, lse = c.attend(workspace, window=90, sinks=2)        # the value is hidden
        bad[0] = False
        assert torch.equal(out.isnan(), bad)


@gpu
def test_infinite_values_in_bf16():
    """Of one sign: the channel is infinite, also where the token's weight is next to nothing; of both:
    NaN.  Hidden ones have no part."""
    _need_gpu()
    c = Case("bf16", 2, 12, 2, 32, [3000, 200], seed=9)
    c.pool[0, c.table[0, 3], 0, 1, 5, 7] = math.inf
    c.pool[0, c.table[0, 80], 0, 1, 5, 8] = -math.inf
    c.pool[1, c.table[1, 1], 1, 1, 5, 9] = math.inf
    c.pool[1, c.table[1, 3], 1, 1, 6, 9] = -math.inf
    for workspace in (False, True):
        out, _ = c.attend(workspace)
        want = torch.zeros_like(out)
        want[0, 0, :6, 7], want[0, 0, :6, 8], want[1, 1, 6:, 9] = math.inf, -math.inf, math.nan
        odd = ~out.isfinite()
        assert torch.equal(odd, (want != 0) | want.isnan())
        assert torch.equal(out[odd].nan_to_num(nan=5.0, posinf=6.0, neginf=7.0), want[odd].nan_to_num(nan=5.0, posinf=6.0, neginf=7.0))
        out, _ = c.attend(workspace, window=99, sinks=30)         # the last one alone is visible
        assert (out[1, 1, 6:, 9] == -math.inf).all() and int((~out.isfinite()).sum()) == 6


@gpu
def test_long_rows_of_few_heads():
    """Rows that are split over many CTAs, next to short and empty ones, at the limit of a sequence."""
    _need_gpu()
    for lengths in ([262144], [100000, 5, 0, 70000]):
        c = Case("e4m3", 1, 4, 1, 16, lengths, seed=10, spare=0)
        a, b = c.attend(), c.attend(workspace=True)
        c.check(*a)
        c.check(*b)
        again = c.attend(workspace=True)
        assert torch.equal(b[0], again[0]) and torch.equal(b[1], again[1])
        c.check(*c.attend(workspace=True, window=65000, sinks=33), 65000, 33)


@gpu
def test_offsets_beyond_32_bits():
    """The last pages of a pool of 5 GB."""
    _need_gpu()
    c = Case("e4m3", 4, 8, 2, 16, [48], seed=11, spare=0)
    P = 160000
    pool = torch.full((4, P, 2, 2, 16, D), 0x7f, dtype=torch.uint8, device="cuda")
    scales = torch.full((4, P, 2, 2, 1), math.nan, device="cuda")
    to = torch.tensor([P - 1, P - 3, P - 2], device="cuda")
    old = torch.from_numpy(c.table[0, :3]).cuda().long()
    pool[:, to] = c.pool.view(torch.uint8)[:, old]
    scales[:, to] = c.scales[:, old]
    table = torch.zeros_like(c.bt)
    table[0, :3] = to.int()
    out = torch.empty_like(c.q)
    lse = torch.empty((1, 4, 8), device="cuda")
    md.md_attend_cache(c.q, pool, table, c.n, out, scales=scales, lse=lse)
    c.check(out, lse)


@gpu
def test_rows_behind_the_batch_and_raw_bits():
    """q and out as parts of larger tensors: what lies behind is left; pools, queries and outputs as
    raw bits."""
    _need_gpu()
    c = Case("e4m3", 1, 16, 2, 16, [77, 500], seed=12)
    whole = torch.full((4,) + c.q.shape[1:], 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4, 1, 16), 7.0, device="cuda")
    md.md_attend_cache(c.q.view(torch.int16), c.pool.view(torch.uint8), c.bt, list(c.n), whole[:2], scales=c.scales, lse=lse[:2])
    c.check(whole[:2], lse[:2])
    assert (whole[2:] == 7).all() and (lse[2:] == 7).all()


@gpu
def test_two_streams_and_two_graphs():
    """Calls at the same time, each with its workspace, give what they give alone; a captured call
    reads its tensors anew at each replay."""
    _need_gpu()
    cases = [Case(kind, 1, 16, 2, 16, lengths, seed=13 + i) for i, (kind, lengths) in
             enumerate((("e4m3", [90000]), ("bf16", [30000, 70]), ("e4m3", [60000, 100])))]
    alone = [c.attend(workspace=True) for c in cases]
    ws = [torch.full((md.MD_ATTEND_WORKSPACE,), 255, dtype=torch.uint8, device="cuda") for _ in cases]
    got = [(torch.zeros_like(o), torch.zeros_like(z)) for o, z in alone]
    streams, graphs = [torch.cuda.Stream() for _ in cases], []

    def call(i, **kw):
        c = cases[i]
        md.md_attend_cache(c.q, c.pool, c.bt, c.n, got[i][0], scales=c.scales, lse=got[i][1], workspace=ws[i], **kw)

    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(3):
            call(i, stream=streams[i])
    torch.cuda.synchronize()
    for i in range(3):
        assert torch.equal(got[i][0], alone[i][0]) and torch.equal(got[i][1], alone[i][1])
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            call(i)
        got[i][0].zero_()
    for c in cases:
        c.q.mul_(-0.5)
    want = [c.attend(workspace=True) for c in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(3):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        assert torch.equal(got[i][0], want[i][0]) and torch.equal(got[i][1], want[i][1])


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_tables_and_pools_that_change_between_calls(kind):
    """Call after call without a wait, the tables, rows and queries rewritten in between: each call sees
    what was there when it was its turn."""
    _need_gpu()
    c = Case(kind, 1, 16, 2, 16, [2000, 300, 17], seed=20)
    tables, got = [c.bt], []
    for i in range(5):                                            # the same pages, others' places; some outside
        t = c.bt.clone()
        t[0, :125] = t[0, torch.randperm(125, device="cuda")]
        t[1, i] = (-1, c.P, 1 << 30, -9, c.P + 5)[i]
        tables.append(t)
    qs = [torch.randn_like(c.q) for _ in tables]
    now, q = c.bt.clone(), c.q.clone()
    torch.cuda.synchronize()
    for t, x in zip(tables * 2, qs * 2):
        out, lse = torch.empty_like(q), torch.empty((3, 1, 16), device="cuda")
        md.md_attend_cache(q, c.pool, now, c.n, out, scales=c.scales, lse=lse)     # busy with the one before
        now.copy_(t)
        q.copy_(x)
        out, lse = torch.empty_like(q), torch.empty((3, 1, 16), device="cuda")
        md.md_attend_cache(q, c.pool, now, c.n, out, scales=c.scales, lse=lse)
        got.append((t, x, out, lse))
    for t, x, out, lse in got:
        c.table, c.q = t.cpu().numpy(), x
        c.check(out, lse)


@gpu
@pytest.mark.parametrize("ps", [16, 32])
def test_a_decode_loop_on_an_eight_bit_cache(ps):
    """Rows from a projection, written as they come (a prompt, then step by step, layer by layer),
    attended under a window, and moved to a bf16 cache in the end."""
    _need_gpu()
    L, Hq, Hkv, B = 2, 12, 2, 3
    g = torch.Generator(device="cuda").manual_seed(ps)
    W = -(-230 // ps)
    P = B * W
    table = torch.randperm(P, generator=g, device="cuda").int().view(B, W)
    pool = torch.full((L, P, Hkv, 2, ps, D), math.nan, device="cuda").to(torch.float8_e4m3fn)
    scales = torch.full((L, P, Hkv, 2, ps // 16), math.nan, device="cuda")
    n = np.array([200, 0, 31], np.int32)
    k, v = (torch.randn((L, Hkv, int(n.sum()), D), generator=g, device="cuda").bfloat16().permute(2, 0, 1, 3) for _ in range(2))
    md.md_write_cache8(k, v, pool, scales, table, np.zeros(3, np.int32), n)
    kept = [[(k[:200], v[:200])], [], [(k[200:], v[200:])]]
    table_rope = md.md_rope_table(np.exp(np.arange(64) * (-np.log(1e6) / 64)), 4096)
    lse = torch.empty((B, 1, Hq), device="cuda")
    for step in range(25):
        new = [[], []]
        for l in range(L):
            x = torch.randn((B, Hq + 2 * Hkv, D), generator=g, device="cuda").bfloat16() * (1 + step % 4)
            q, kk, vv = (torch.empty((B, 1, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
            md.md_norm_rope(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], q[:, 0], kk[:, 0], vv[:, 0],
                            positions=torch.from_numpy(n).cuda(), table=table_rope,
                            q_weight=torch.ones(D, device="cuda"), k_weight=torch.ones(D, device="cuda"))
            md.md_write_cache8(kk, vv, pool[l:l + 1], scales[l:l + 1], table, n, np.ones(3, np.int32))
            out = torch.empty_like(q)
            md.md_attend_cache(q, pool[l:l + 1], table, n + 1, out, scales=scales[l:l + 1], window=64, sinks=4, lse=lse)
            c = Case.__new__(Case)
            c.kind, c.L, c.Hq, c.Hkv, c.ps, c.G, c.B, c.P, c.n = "e4m3", 1, Hq, Hkv, ps, Hq // Hkv, B, P, n + 1
            c.table, c.pool, c.scales, c.q = table.cpu().numpy(), pool[l:l + 1], scales[l:l + 1], q
            c.check(out, lse, 64, 4)
            new[0].append(kk)
            new[1].append(vv)
        for b in range(B):
            kept[b].append((torch.cat([x[b:b + 1] for x in new[0]], 1), torch.cat([x[b:b + 1] for x in new[1]], 1)))
        n = n + 1
    k, v = (torch.empty((L, Hkv, int(n.sum()), D), dtype=torch.bfloat16, device="cuda").permute(2, 0, 1, 3) for _ in range(2))
    md.md_read_cache8(k, v, pool, scales, table, np.zeros(3, np.int32), n)
    at = 0
    for b in range(B):
        for got, i in ((k, 0), (v, 1)):
            want = torch.cat([x[i] for x in kept[b]]).float()
            err = (got[at:at + n[b]].float() - want).abs()
            # e4m3: half a step, 2^-4 of the value, twice where a block moved to a larger scale and the code became
            # subnormal: 2^-10 of a scale each, and the scale is at most 2 / 448 of the block's largest value
            assert (err <= 2.0 ** -4 * want.abs() + 2 * 2.0 ** -10 * 2 / 448 * want.abs().amax()).all()
        at += n[b]


# ------------------------------------------------------------- refusals, on the CPU ----
def _args(**kw):
    a = md.md_attend_cache_args()
    at = 1 << 20
    d = dict(batch=2, num_layers=2, num_q_heads=8, num_kv_heads=2, page_size=16, max_pages_per_seq=4, num_phys_pages=9,
             type=md.MD_TYPE_E4M3, window=-1, sinks=0, q_dev=at, pool_dev=at, scales_dev=at, block_table_dev=at,
             n_tokens_host=[20, 0], out_dev=at, lse_dev=None, workspace_dev=None, workspace_bytes=0, stream=None)
    d.update(kw)
    if d["n_tokens_host"] is not None:
        a.hold = np.array(d["n_tokens_host"], np.int32)
        d["n_tokens_host"] = a.hold.ctypes.data
    for n, x in d.items():
        setattr(a, n, x)
    return a


AT = 1 << 20
REFUSED = [dict(batch=0), dict(batch=257), dict(num_layers=0), dict(num_layers=256), dict(num_q_heads=0),
           dict(num_q_heads=9), dict(num_q_heads=18), dict(num_q_heads=1), dict(num_kv_heads=0), dict(page_size=8),
           dict(page_size=64), dict(max_pages_per_seq=0), dict(max_pages_per_seq=1 << 15), dict(num_phys_pages=0),
           dict(num_phys_pages=1 << 27), dict(type=md.MD_TYPE_F16), dict(type=md.MD_TYPE_F32), dict(type=4), dict(type=-1),
           dict(window=-2), dict(sinks=-1), dict(q_dev=None), dict(q_dev=AT + 8), dict(pool_dev=None),
           dict(pool_dev=AT + 8), dict(scales_dev=None), dict(scales_dev=AT + 2), dict(block_table_dev=None),
           dict(block_table_dev=AT + 2), dict(n_tokens_host=None), dict(n_tokens_host=[65, 0]), dict(n_tokens_host=[-1, 0]),
           dict(out_dev=None), dict(out_dev=AT + 4), dict(lse_dev=AT + 2)]


@pytest.mark.parametrize("bad", REFUSED, ids=[",".join(x) + str(i) for i, x in enumerate(REFUSED)])
def test_arguments_are_refused_before_any_launch(bad):
    assert md.lib().md_attend_cache(ctypes.byref(_args(**bad))) == md.MD_ERR_INVALID_ARG
    assert md.lib().md_attend_cache(None) == md.MD_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(workspace_dev=AT, workspace_bytes=md.MD_ATTEND_WORKSPACE - 1),
                                 dict(workspace_dev=AT + 8, workspace_bytes=md.MD_ATTEND_WORKSPACE)])
def test_workspaces_are_refused_before_any_launch(bad):
    assert md.lib().md_attend_cache(ctypes.byref(_args(**bad))) == md.MD_ERR_WORKSPACE
