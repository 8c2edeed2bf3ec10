"""md_attend_cache looks up its first pages while the launch before it ends.  Here that launch is the library's own
and rewrites the block table: it lets the attention start early, and ends with the table's rows.  Each call must
work with the table behind it, whatever it saw ahead of it."""
import numpy as np
import pytest

import paper_2607_10582_gb300 as md
from tests.test_attend_cache import Case, _need_gpu

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
WIDTH = 128                                                       # entries of a row of the table: a row of the cache
# Rows that are read before the table's: all CTAs of that launch run at once, two to an SM, and so let the attention
# start while they wait for their rows.  Four in ten of its early look-ups then see the table before this one (none do
# with 3,000 rows, where the launch is over too soon, or with 60,000, where the SMs are full until it is).
FILL = 30000


class Tables:
    """Block tables [batch][128] that md_read_cache8 writes as fp32 rows: an entry i is the bits of i x 2^-149, code i
    under a scale of 2^-149; a negative code gives an entry far below 0."""

    def __init__(self, tables):
        B = tables[0].shape[0]
        blocks = -(-B // 16)
        self.codes, pages = [], 1 + blocks
        self.scales = torch.full((1, pages, 1, 2, 1), float(np.uint32(1).view(np.float32)), device="cuda")
        for t in tables:
            x = torch.zeros((1, pages, 1, 2, 16, WIDTH))
            for b in range(B):
                x[0, 1 + b // 16, 0, 0, b % 16] = torch.from_numpy(t[b]).float()
            c = x.to(torch.float8_e4m3fn)
            assert torch.equal(c.float(), x)                      # page ids that a code holds
            self.codes.append(c.cuda())
        self.bt = torch.zeros((2, max(FILL // 16 + 1, blocks)), dtype=torch.int32, device="cuda")
        self.bt[1, :blocks] = torch.arange(1, pages, device="cuda")
        self.k, self.v = (torch.zeros((FILL + B, 1, 1, WIDTH), device="cuda") for _ in range(2))
        self.table = self.k[FILL:, 0, 0].view(torch.int32)
        self.count = np.array([FILL, B], np.int32)

    def put(self, i):
        md.md_read_cache8(self.k, self.v, self.codes[i], self.scales, self.bt, np.zeros(2, np.int32), self.count)


def _cases(kind):
    """Caches whose page ids codes hold, and tables over them: one as it is, others with the pages in other
    places, and with entries outside the pool."""
    c = Case(kind, 1, 16, 2, 32, [100, 230, 0, 96, 200], seed=50, spare=0)
    assert c.P <= 24
    ids = np.array([i if i <= 16 else 2 * i - 16 for i in range(c.P)])           # even above 16: codes hold them
    P = int(ids.max()) + 1
    pool = torch.full((1, P) + c.pool.shape[2:], float("nan"), device="cuda").to(c.pool.dtype)
    raw = torch.uint8 if kind == "e4m3" else torch.int16
    to = torch.from_numpy(ids).cuda()
    pool.view(raw)[:, to] = c.pool.view(raw)
    if c.scales is not None:
        scales = torch.full((1, P) + c.scales.shape[2:], float("nan"), device="cuda")
        scales[:, to] = c.scales
        c.scales = scales
    c.pool, c.P = pool, P
    r = np.random.default_rng(51)
    tables = []
    for i in range(3):
        t = np.full((c.B, WIDTH), -1, np.int32)                   # behind the pages: outside
        for b in range(c.B):
            at = ids[c.table[b, :c.pages[b]]]
            full = c.n[b] // 32                                   # the last page, if not full, stays the last
            t[b, :c.pages[b]] = np.concatenate([r.permutation(at[:full]), at[full:]])
            if i and full:
                t[b, r.integers(full)] = (-3, 320)[i - 1]
        tables.append(t)
    return c, tables


@pytest.mark.parametrize("code", [0, 1, 7, 16, 18, 32, 320])
def test_a_code_times_the_smallest_scale_is_a_page_id(code):
    x = torch.tensor([float(code)]).to(torch.float8_e4m3fn).double() * 2.0 ** -149
    assert int(x.float().view(torch.int32)) == code


@gpu
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_a_table_that_the_launch_before_writes(kind, graph):
    _need_gpu()
    c, tables = _cases(kind)
    t = Tables(tables)
    want = []
    for i, x in enumerate(tables):                                # one at a time, against the 64-bit reference
        t.put(i)
        torch.cuda.synchronize()
        got = t.table.cpu().numpy()
        assert np.array_equal(np.where(x < 0, 0, x), np.where(x < 0, 0, got)) and (got[x < 0] < 0).all()
        out, lse = torch.empty_like(c.q), torch.empty((c.B, 1, c.Hq), device="cuda")
        md.md_attend_cache(c.q, c.pool, t.table, c.n, out, scales=c.scales, lse=lse)
        torch.cuda.synchronize()
        c.table, c.W = x, WIDTH
        c.check(out, lse)
        want.append((out, lse))
    assert not torch.equal(want[0][0], want[1][0]) and not torch.equal(want[0][0], want[2][0])
    order = np.random.default_rng(52).integers(0, 3, 60)
    outs = [(torch.empty_like(c.q), torch.empty((c.B, 1, c.Hq), device="cuda")) for _ in order]

    def loop():
        for i, (out, lse) in zip(order, outs):
            t.put(i)
            md.md_attend_cache(c.q, c.pool, t.table, c.n, out, scales=c.scales, lse=lse)

    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            loop()
    for _ in range(5):
        for out, lse in outs:
            out.fill_(7)
            lse.fill_(7)
        g.replay() if graph else loop()
        torch.cuda.synchronize()
        for i, (out, lse) in zip(order, outs):
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
