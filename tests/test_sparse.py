"""md_sparse_enable: decode steps of a handle over selected pages.

With contiguous pages a step's output is that of the page calls on the handle's own pool
and table, bit for bit, and its mass their masses' sum (for a layer-by-layer step, calls of
one layer each: how a row is split, and so its rounding, goes by a launch's size);
tests/test_pages.py holds those calls to their formulas.  Region-aligned pages are held to the formulas directly, with the
tolerances given there."""
import ctypes
import math

import numpy as np
import pytest

import paper_2607_10582_gb300 as md
from paper_2607_10582_gb300 import build as mdbuild

torch = pytest.importorskip("torch")
D = 128
mdbuild.build()
gpu = pytest.mark.gpu
UNIT = 2.0 ** -48
CHAIN = 18 * 2.0 ** -24


class Loop:
    """A decode loop with its own inputs."""

    def __init__(self, L, Hq, Hkv, ps, lengths, seed=0, room=200, **kw):
        if not torch.cuda.is_available():  # pragma: no cover
            pytest.skip("needs a CUDA GPU")
        self.L, self.Hq, self.Hkv, self.ps, self.B = L, Hq, Hkv, ps, len(lengths)
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        width = max(lengths) // ps + room
        self.c = md.Cache(L, Hq, Hkv, ps, self.B, width, sum(lengths) // ps + self.B * room, **kw)
        for r in range(7):
            self.c.set_region_params(r, 1.0 - 0.1 * r, 20.0 + 10 * r, r == 0)
        for b, n in enumerate(lengths):
            self.append(b, n)

    def rand(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda").bfloat16()

    def append(self, b, n):
        lab = np.sort(self.rng.integers(0, 7, n)).astype(np.uint8)
        self.c.append_tokens(b, lab, self.rand(self.L, self.Hkv, n, D), self.rand(self.L, self.Hkv, n, D))

    def step(self, how="step", q=None, kv=None, regions=None):
        B, L = self.B, self.L
        q = self.rand(B, L, self.Hq, D) if q is None else q
        k, v = (self.rand(B, L, self.Hkv, D) for _ in range(2)) if kv is None else kv
        regions = np.full(B, 6, np.uint8) if regions is None else regions
        out = torch.full_like(q, math.nan)
        if how == "layers":
            for l in range(L):
                o = torch.empty_like(q[:, l])
                self.c.decode_layer(l, B, q[:, l].contiguous(), k[:, l].contiguous(), v[:, l].contiguous(), regions, o)
                out[:, l] = o
        elif how == "host":
            h = torch.empty(q.shape, dtype=q.dtype, pin_memory=True)
            self.c.decode_step_host(B, *(x.cpu().pin_memory() for x in (q, k, v)), regions, h)
            assert self.c.sync() == md.MD_OK
            out = h.cuda()
        else:
            self.c.decode_step(B, q, k, v, regions, out)
        return q, out

    def tokens(self):
        return np.array([self.c.query(md.MD_QUERY_TOKENS, b) for b in range(self.B)], np.int32)

    def pages(self):
        return [self.c.query(md.MD_QUERY_PAGES, b) for b in range(self.B)]

    def by_page_calls(self, q, top, first, last, each_layer):
        """The step just run, by the page calls: output, and mass per slot."""
        pool, bt, n = self.c.get_state(md.MD_STATE_POOL), self.c.get_state(md.MD_STATE_BLOCK_TABLE), self.tokens()
        L, P, W, rows = self.L, pool.shape[1], bt.shape[1], (self.B, self.L, self.Hkv)
        bounds = torch.zeros((L, P, self.Hkv, 2, D), dtype=torch.bfloat16, device="cuda")
        scores = torch.zeros(rows + (W,), device="cuda")
        ids = torch.empty(rows + (top,), dtype=torch.int32, device="cuda")
        out, mass = torch.empty_like(q), torch.empty(rows + (top * self.ps,), device="cuda")
        md.md_page_bounds(pool, bt, n, bounds)
        md.md_page_scores(q, bounds, bt, n, scores, page_size=self.ps)
        md.md_page_top(scores, n, ids, page_size=self.ps, first=first, last=last)
        for l in range(L) if each_layer else [slice(None)]:
            part = slice(l, l + 1) if each_layer else l
            o, m = torch.empty_like(q[:, part]).contiguous(), torch.empty_like(mass[:, part]).contiguous()
            md.md_attend_pages(q[:, part].contiguous(), pool[part], bt, n, ids[:, part].contiguous(), o, mass=m)
            out[:, part], mass[:, part] = o, m
        acc = torch.zeros(P * self.ps, dtype=torch.float64, device="cuda")
        for b in range(self.B):
            i = ids[b].long()
            slot = bt[b, i.clamp(min=0)].long()[..., None] * self.ps + torch.arange(self.ps, device="cuda")
            keep = (i >= 0)[..., None].expand_as(slot)
            acc.index_add_(0, slot[keep], mass[b].double().view(slot.shape)[keep])
        return out, acc

    def check(self, how, top, first=1, last=1):
        q, out = self.step(how)
        mass = self.c.get_state(md.MD_STATE_MASS).double() * UNIT
        want, acc = self.by_page_calls(q, top, first, last, how == "layers")
        assert torch.equal(out, want)
        # each addend is rounded to 2^-48
        assert (mass - acc).abs().max() <= self.L * self.Hkv * 2.0 ** -48 + 2.0 ** -50 * self.L * self.Hq
        assert abs(float(mass.sum()) - self.B * self.L * self.Hq) < 1e-3 * self.B * self.L * self.Hq


@gpu
@pytest.mark.parametrize("how", ["step", "layers", "host"])
@pytest.mark.parametrize("L,Hq,Hkv,ps,lengths,top,first,last", [
    (1, 12, 2, 16, [448], 6, 1, 1),
    (3, 16, 2, 32, [900, 20, 3000], 17, 2, 3),
    (2, 8, 4, 16, [1700, 1500, 40, 1], 24, 0, 1),
])
def test_steps_attend_the_selected_pages(L, Hq, Hkv, ps, lengths, top, first, last, how):
    """Steps that fill pages, appends and evictions in between."""
    s = Loop(L, Hq, Hkv, ps, lengths, seed=top)
    s.c.sparse_enable(top, first, last)
    for i in range(2 * ps + 3):
        if i % 11 in (0, 1, 7) or s.ps - 2 <= i % s.ps:
            s.check(how, top, first, last)
        else:
            s.step(how)
        if i % 5 == 4:
            s.c.evict(np.array([max(top + 2, p - 2) for p in s.pages()], np.int32))
        if i % 13 == 12:
            s.append(i % s.B, 70)
    assert s.c.sync() == md.MD_OK


@gpu
def test_short_sequences_are_attended_in_full():
    """No sequence above top_pages: the step is the one without a selection, bit for bit;
    the same for a handle whose selection was turned off."""
    L, lengths = 2, [300, 77]
    a, b, c = (Loop(L, 16, 2, 16, lengths, seed=4) for _ in range(3))
    a.c.sparse_enable(25)
    c.c.sparse_enable(3)
    c.c.sparse_enable(0)
    for how in ("step", "layers", "host"):
        outs = [x.step(how)[1] for x in (a, b, c)]
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        assert torch.equal(a.c.get_state(md.MD_STATE_MASS), b.c.get_state(md.MD_STATE_MASS))


@gpu
def test_selecting_all_but_nothing_changes_the_sum():
    """Just above the threshold: one page of many is left out; and sparse and dense steps
    may alternate, pages filled under dense steps being bounded when they are needed."""
    s = Loop(2, 16, 2, 16, [640 + 5], seed=5)
    for i in range(40):
        if i % 3 == 2:
            s.c.sparse_enable(0)
            s.step()
        elif i % 3 == 0:
            s.c.sparse_enable(s.pages()[0] - 1)
            s.check("step", s.pages()[0] - 1) if s.tokens()[0] % 16 else s.step()
        else:
            s.c.sparse_enable(7)
            s.check("layers", 7)


@gpu
def test_eviction_observes_the_selected_tokens():
    """Pages that were not attended have no mass, and go first under pure accumulation."""
    s = Loop(1, 8, 1, 16, [1600], seed=6, rho=1.0, gamma=1.0, attn_weight=1.0)
    for r in range(7):
        s.c.set_region_params(r, 0.0, math.inf, r == 0)
    s.c.sparse_enable(30)
    q, _ = s.step()
    mass = s.c.get_state(md.MD_STATE_MASS).view(-1, 16).sum(1)
    table = s.c.get_state(md.MD_STATE_BLOCK_TABLE)[0, :101].long()
    pinned = s.c.query(md.MD_QUERY_PINNED_PAGES, 0)
    seen = mass[table] > 0
    assert int(seen.sum()) == 30
    unseen = [int(x) for x in table[~seen]]
    ids = torch.empty((1, s.c.P_max), dtype=torch.int32, device="cuda")
    s.c.evict([101 - 20], ids)
    gone = [int(x) for x in ids[0] if x >= 0]
    assert len(gone) == 20 and set(gone) <= set(unseen) and pinned < 101 - 30
    s.check("step", 30)


@gpu
def test_checkpoint_under_selection():
    s = Loop(2, 16, 2, 16, [700, 300], seed=7)
    s.c.sparse_enable(9)
    s.step()
    s.c.evict([40, 20])
    saved = s.c.save_state()
    q, k, v = s.rand(2, 2, 16, D), s.rand(2, 2, 2, D), s.rand(2, 2, 2, D)
    _, first = s.step(q=q, kv=(k, v))
    s.c.evict([39, 19])
    s.c.load_state(saved)
    _, again = s.step(q=q, kv=(k, v))
    assert torch.equal(first, again)
    for _ in range(20):
        s.check("step", 9)


@gpu
@pytest.mark.parametrize("ps", [16, 32])
def test_region_aligned_pages(ps):
    """Partly filled pages in the middle: one layer and KV head, so that the mass shows the
    pages attended."""
    s = Loop(1, 8, 1, ps, [900], seed=8, region_aligned_pages=1)
    top = 11
    s.c.sparse_enable(top, 1, 2)
    for i in range(45):
        q, out = s.step(regions=np.array([(i // 5) % 7], np.uint8))
        n = s.pages()[0]
        table = s.c.get_state(md.MD_STATE_BLOCK_TABLE)[0, :n].long()
        fill = s.c.get_state(md.MD_STATE_PAGE_FILL)[0, :n].long()
        pool = s.c.get_state(md.MD_STATE_POOL).view(torch.bfloat16)[0, table, 0].double()   # [n][2][ps][D]
        mass = s.c.get_state(md.MD_STATE_MASS).double().view(-1, ps)[table] * UNIT
        held = torch.arange(ps, device="cuda") < fill[:, None]
        k, v = pool[:, 0], torch.where(held[..., None], pool[:, 1], 0)
        hi = torch.where(held[..., None], k, -math.inf).amax(1)
        lo = torch.where(held[..., None], k, math.inf).amin(1)
        x = q[0, 0].double()
        bound = (x.clamp(min=0) @ hi.T + x.clamp(max=0) @ lo.T).amax(0) / math.sqrt(D)
        seen = mass.sum(1) > 0
        assert int(seen.sum()) == top and seen[0] and seen[-2:].all()
        slack = 16 * CHAIN * float((x.abs() @ torch.maximum(hi.abs(), lo.abs()).T).max()) / math.sqrt(D)
        mid = slice(1, n - 2)
        assert bound[mid][seen[mid]].min() >= bound[mid][~seen[mid]].max() - 2 * slack
        use = (held & seen[:, None]).flatten()
        kk, vv = k.flatten(0, 1)[use], v.flatten(0, 1)[use]
        p = torch.softmax(x @ kk.T / math.sqrt(D), -1)
        delta = 8 * CHAIN * float((x.abs() @ kk.abs().T).max()) / math.sqrt(D)
        ref = p @ vv
        tol = 2.0 ** -8 * ref.abs() + (2 * delta + 2.0 ** -15) * (p @ vv.abs())
        assert ((out[0, 0].double() - ref).abs() <= tol).all()
        assert ((mass.flatten()[use] - p.sum(0)).abs() <= (2 * delta + 2.0 ** -18) * p.sum(0) + 8 * UNIT).all()
        assert not mass.flatten()[~use].any()
        if i % 6 == 5:
            s.c.evict([max(20, n - 3)])


@gpu
def test_wait_limit_shorter_than_a_copy():
    """A copy that does not land within the handle's limit ends the step with a status, and what
    was in flight lands before the launch ends: a new handle works."""
    s = Loop(2, 16, 2, 32, [3000, 500], seed=10)
    s.c.sparse_enable(40)
    s.c.debug_set(md.MD_DEBUG_SPIN_LIMIT_NS, 1000)
    statuses = set()
    for _ in range(30):
        s.step()
        statuses.add(s.c.sync())
        if md.MD_ERR_DEVICE_TIMEOUT in statuses:
            break
    assert statuses <= {md.MD_OK, md.MD_ERR_DEVICE_TIMEOUT}
    if md.MD_ERR_DEVICE_TIMEOUT in statuses:
        with pytest.raises(md.MemDecayError):
            s.step()
    t = Loop(2, 16, 2, 32, [3000, 500], seed=10)
    t.c.sparse_enable(40)
    t.check("step", 40)


@gpu
def test_wait_limit_with_lists_of_many_tiles():
    """A row that gives up early in a list of hundreds, most entries of which are no pages: its
    masses go to tokens of the list only, and a new handle works."""
    lengths = [6000] * 30 + [40, 17]
    s = Loop(2, 16, 2, 16, lengths, seed=12)
    s.c.sparse_enable(300)
    s.c.debug_set(md.MD_DEBUG_SPIN_LIMIT_NS, 1000)
    for _ in range(30):
        s.step()
        if s.c.sync() == md.MD_ERR_DEVICE_TIMEOUT:
            break
    t = Loop(2, 16, 2, 16, lengths, seed=12)
    t.c.sparse_enable(300)
    t.check("step", 300)


@gpu
@pytest.mark.parametrize("how", ["step", "layers"])
def test_queries_and_outputs_at_any_address(how):
    """Rows that start at any 2-byte address give the same bits, and nothing around the outputs
    is written."""
    want = None
    for q_shift, out_shift in ((0, 0), (0, 1), (0, 2), (0, 4), (1, 0), (2, 4), (4, 3), (8, 8)):
        s = Loop(2, 16, 2, 16, [700, 90, 1300], seed=16)
        s.c.sparse_enable(9)
        q, k, v = s.rand(3, 2, 16, D), s.rand(3, 2, 2, D), s.rand(3, 2, 2, D)
        outs = []
        for l in range(2) if how == "layers" else [slice(None)]:
            x, kk, vv = (y[:, l].contiguous() for y in (q, k, v))
            src = torch.zeros(x.numel() + 16, dtype=torch.bfloat16, device="cuda")
            src[q_shift:q_shift + x.numel()] = x.flatten()
            dst = torch.zeros(x.numel() + 16, dtype=torch.int16, device="cuda")
            at = (src.data_ptr() + 2 * q_shift, kk, vv, [6] * 3, dst.data_ptr() + 2 * out_shift)
            s.c.decode_layer(l, 3, *at) if how == "layers" else s.c.decode_step(3, *at)
            assert s.c.sync() == md.MD_OK
            assert not dst[:out_shift].any() and not dst[out_shift + x.numel():].any()
            outs.append(dst[out_shift:out_shift + x.numel()])
        outs = torch.cat(outs)
        want = outs if want is None else want
        assert torch.equal(outs, want) and outs.any()


@gpu
def test_enabled_from_another_stream_with_work_pending():
    """A block that the current stream has given up, with writes to it pending, is no buffer of a
    handle on another stream before those writes are done."""
    if not torch.cuda.is_available():  # pragma: no cover
        pytest.skip("needs a CUDA GPU")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s = Loop(2, 16, 2, 16, [900, 400], seed=17, stream=side)
    n = int(md.lib().md_sparse_bytes(ctypes.byref(s.c.cfg), 9)) + 256
    old = torch.empty(n, dtype=torch.uint8, device="cuda")
    big = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for _ in range(100):
        big.fill_(1)                               # some ms
    old.fill_(0)
    del old
    s.c.sparse_enable(9)
    with torch.cuda.stream(side):
        for _ in range(3):
            s.check("step", 9)
        torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
        s.check("step", 9)


@gpu
def test_infinite_values_stay_infinite():
    """As in the step over all pages."""
    outs = []
    for top in (0, 12):
        s = Loop(2, 16, 2, 16, [190], seed=18)
        s.c.sparse_enable(top, 1, 2)                         # the infinity's page is the last but one
        q, k, v = s.rand(1, 2, 16, D), s.rand(1, 2, 2, D), s.rand(1, 2, 2, D)
        v[0, 1, 0, 9] = math.inf
        s.step(q=q, kv=(k, v))
        s.step(q=q, kv=(k, torch.zeros_like(v)))
        s.step(q=q, kv=(k, torch.zeros_like(v)))             # the 193rd token: a 13th page
        outs.append(s.step(q=q, kv=(k, torch.zeros_like(v)))[1])
    want = torch.zeros_like(outs[0], dtype=torch.bool)
    want[0, 1, :8, 9] = True
    assert s.pages() == [13] and all(torch.equal(o.isinf(), want) and not o.isnan().any() for o in outs)


@gpu
@pytest.mark.parametrize("lengths,top,tile", [
    ([3000, 500], 40, 0),                          # clusters of CTAs over a row
    ([6000] * 30 + [40, 17], 300, 0),              # one CTA per row, scores in tensor memory; lists of hundreds,
    ([6000] * 30 + [40, 17], 300, 5),              # of the last two sequences' most entries are no pages
    ([6000] * 30 + [40, 17], 300, 33),             # in the second list of 32
])
def test_a_row_that_gives_up(lengths, top, tile):
    """A copy taken for one that did not land: the step reports it, the row's outputs are NaN and
    the others' are not, no state but the mass of the listed tokens is written, and a new handle
    works."""
    s = Loop(2, 16, 2, 16, lengths, seed=19)
    s.c.sparse_enable(top)
    s.step()
    assert s.c.evict(np.array(s.pages(), np.int32))[0] == md.MD_OK and s.c.sync() == md.MD_OK
    # the new tokens' own slots start with the step
    state = {w: s.c.get_state(w).clone() for w in (md.MD_STATE_TOKEN_PRIO, md.MD_STATE_WINDOW, md.MD_STATE_AHAT)}
    n = s.tokens()
    s.c.debug_set(md.MD_DEBUG_LOST_TILE, tile)
    q, out = s.step()
    assert s.c.sync() == md.MD_ERR_DEVICE_TIMEOUT
    with pytest.raises(md.MemDecayError):
        s.step()
    want, acc = s.by_page_calls(q, top, 1, 1, False)
    nan = out.isnan()
    gone = nan.all(-1)
    assert torch.equal(gone, nan.any(-1)) and torch.equal(torch.where(nan, 0, out), torch.where(nan, 0, want))
    short = [b for b, x in enumerate(lengths) if x < 100]
    assert gone.all() if tile == 0 else gone.any() and not gone[short].any()
    mass = s.c.get_state(md.MD_STATE_MASS)
    listed = acc > 0
    assert not mass[~listed].any()
    table = s.c.get_state(md.MD_STATE_BLOCK_TABLE)
    new = torch.tensor([int(table[b, x // 16]) * 16 + x % 16 for b, x in enumerate(n)], device="cuda")
    for w, before in state.items():
        now = s.c.get_state(w)
        now[new] = before[new]
        assert torch.equal(now.view(torch.int32), before.view(torch.int32)), w
    t = Loop(2, 16, 2, 16, lengths, seed=19)
    t.c.sparse_enable(top)
    t.check("step", top)


@gpu
def test_refusals_leave_the_handle_as_it_was():
    s = Loop(2, 16, 2, 16, [400], seed=9)
    for top, first, last in ((-1, 1, 1), (5000, 1, 1), (4, 1, 0), (4, -1, 1), (4, 3, 2), (4, 5, 1)):
        with pytest.raises(md.MemDecayError) as e:
            s.c.sparse_enable(top, first, last)
        assert e.value.status == md.MD_ERR_INVALID_ARG
    lib, need = md.lib(), int(md.lib().md_sparse_bytes(ctypes.byref(s.c.cfg), 4))
    buf = torch.empty(need + 512, dtype=torch.uint8, device="cuda")
    at = (buf.data_ptr() + 255) // 256 * 256
    for p, n in ((None, need), (at + 16, need), (at, need - 1)):
        assert lib.md_sparse_enable(s.c.h, 4, 1, 1, p, n) == md.MD_ERR_WORKSPACE
    q, k = s.rand(1, 16, D), s.rand(1, 2, D)
    s.c.decode_layer(0, 1, q, k, k, [6], torch.empty_like(q))
    assert lib.md_sparse_enable(s.c.h, 4, 1, 1, at, need) == md.MD_ERR_STATE
    s.c.decode_layer(1, 1, q, k, k, [6], torch.empty_like(q))
    s.c.sparse_enable(4)
    s.check("step", 4)


def test_buffer_size_is_host_arithmetic():
    cfg = md.md_config(2, 16, 2, 128, 16, 4, 64, 256, 0.9, 0.1, 2.0, 1.0, 0, 0, 1, None, 0, None, 0, 0)
    size = lambda top: int(md.lib().md_sparse_bytes(ctypes.byref(cfg), top))  # noqa: E731
    assert size(8) >= 2 * 256 * 2 * 512 + 4 * 4 * 64 * 4 + 4 * 4 * 8 * 4
    assert size(0) == size(-1) == size(md.MD_MAX_TOP_TOKENS // 16 + 1) == 0 and size(64) > size(8)
    cfg.page_size = 8
    assert size(8) == 0 and int(md.lib().md_sparse_bytes(None, 8)) == 0
    assert md.lib().md_sparse_enable(None, 0, 0, 0, None, 0) == md.MD_ERR_INVALID_ARG
