"""A cache in eight bits: what md_write_cache8 stores and md_read_cache8 gives back, against a plain
64-bit implementation.  Both are exact, bit for bit: a scale is a power of two, so that the quotient by it is
exact and each code is rounded once (twice where a block moves to a larger scale, which the
reference does as well)."""
import ctypes
import math

import numpy as np
import pytest

import paper_2607_10582_gb300 as md
from paper_2607_10582_gb300 import build as mdbuild

torch = pytest.importorskip("torch")
D, BLOCK = 128, 16
mdbuild.build()
gpu = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# the values of the codes 0 .. 126, by the format's definition
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)])[:127]


def _need_gpu():
    if not torch.cuda.is_available():  # pragma: no cover
        pytest.skip("needs a CUDA GPU")


def encode(x):
    """Codes of float64 values: the nearest, ties to the even code; NaN (0x7f) for what is not finite."""
    size = np.abs(x)
    with np.errstate(invalid="ignore"):
        at = np.clip(np.searchsorted(E4M3, np.where(np.isfinite(x), size, 0)), 1, 126)
        lo, hi = E4M3[at - 1], E4M3[at]
        up = (size - lo > hi - size) | ((size - lo == hi - size) & (at % 2 == 0))
    code = np.where(up, at, at - 1) | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def decode(c):
    v = np.append(E4M3, math.nan)[c & 127]
    return np.where(c & 128, -v, v)


def scale_of(x):
    """The least power of two s, 2^-126 at least, with |x| <= 448 s for the finite values."""
    size = np.abs(x[np.isfinite(x)])
    most = float(size.max()) if size.size else 0.0
    s = 2.0 ** -126
    while most > 448 * s:
        s *= 2
    return s


def write_ref(codes, scales, k, v, table, first, count):
    """codes uint8 [L][P][Hkv][2][ps][D] and scales float64 [L][P][Hkv][2][ps / 16], written in place."""
    L, P, Hkv, _, ps, _ = codes.shape
    row = 0
    for b in range(len(first)):
        for block in range(first[b] // BLOCK, -(-(first[b] + count[b]) // BLOCK) if count[b] else 0):
            lo, hi = max(first[b], block * BLOCK), min(first[b] + count[b], (block + 1) * BLOCK)
            phys, part = table[b, block * BLOCK // ps], block * BLOCK % ps // BLOCK
            if not 0 <= phys < P:
                continue
            for l in range(L):
                for h in range(Hkv):
                    for which, x in enumerate((k, v)):
                        new = x[row + lo - first[b]:row + hi - first[b], l, h]
                        c = codes[l, phys, h, which, part * BLOCK:(part + 1) * BLOCK]
                        s, at = scale_of(new), lo - block * BLOCK
                        if at:
                            was = scales[l, phys, h, which, part]
                            if s > was:
                                c[:at] = encode(decode(c[:at]) * (was / s))
                            s = max(s, was)
                        c[at:at + hi - lo] = encode(new / s)
                        scales[l, phys, h, which, part] = s
        row += count[b]


class Store:
    """A cache in eight bits on the GPU and its reference on the host, junk where nothing was written."""

    def __init__(self, L, Hkv, ps, batch, width, seed, spare=2):
        rng = np.random.default_rng(seed)
        self.rng, self.L, self.Hkv, self.ps, self.B = rng, L, Hkv, ps, batch
        self.P = batch * width + spare
        self.table = rng.permutation(self.P)[:batch * width].reshape(batch, width).astype(np.int32)
        self.codes = rng.integers(0, 256, (L, self.P, Hkv, 2, ps, D)).astype(np.uint8)
        self.scales = rng.choice([math.nan, 0.0, 1.0, -3.0, math.inf], (L, self.P, Hkv, 2, ps // BLOCK))
        self.n = [0] * batch
        self.to_gpu()

    def to_gpu(self):
        self.pool = torch.from_numpy(self.codes).cuda()
        self.sc = torch.from_numpy(self.scales.astype(np.float32)).cuda()
        self.bt = torch.from_numpy(self.table).cuda()

    def rows(self, n, kind, size=1.0, layout="rows"):
        """k and v of n tokens in one of the layouts that callers have."""
        L, Hkv = self.L, self.Hkv
        out = []
        for _ in range(2):
            x = torch.from_numpy(self.rng.standard_normal((n, L, Hkv, D)) * size).to(TYPES[kind]).cuda()
            if layout == "prompt":                                # [L][Hkv][n][D]
                x = x.permute(1, 2, 0, 3).contiguous().permute(2, 0, 1, 3)
            elif layout == "part":                                # of a wider projection, rows apart
                w = torch.zeros((n, L, 3 * Hkv + 1, D + 4), dtype=x.dtype, device="cuda")
                w[:, :, 1:1 + Hkv, :D] = x
                x = w[:, :, 1:1 + Hkv, :D]
            out.append(x)
        return out

    def write(self, k, v, count, **kw):
        first = np.array(self.n, np.int32)
        count = np.array(count, np.int32)
        md.md_write_cache8(k, v, self.pool, self.sc, self.bt, first, count, **kw)
        write_ref(self.codes, self.scales, k.double().cpu().numpy(), v.double().cpu().numpy(), self.table, first, count)
        self.n = [a + int(c) for a, c in zip(self.n, count)]

    def check(self):
        off = np.argwhere(self.pool.cpu().numpy() != self.codes)
        assert not len(off), (len(off), off[:5].tolist())
        want = self.scales.astype(np.float32)
        assert np.array_equal(self.sc.cpu().numpy(), want, equal_nan=True)


def test_the_reference_rounds_like_the_format():
    """The codes of every e4m3 value are itself, and the middle of two goes to the even one."""
    c = np.arange(127, dtype=np.uint8)
    assert np.array_equal(encode(decode(c)), c) and np.array_equal(encode(decode(c | 128)), c | 128)
    mid = (E4M3[1:] + E4M3[:-1]) / 2
    assert np.array_equal(encode(mid), np.where(c[:-1] % 2 == 0, c[:-1], c[1:]))
    x = torch.from_numpy(np.random.default_rng(0).standard_normal(4096) * 60).clamp(-448, 448)
    assert np.array_equal(encode(x.numpy()), x.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()) or \
        (x.float().double() != x).any()
    assert encode(np.array([math.inf, -math.inf, math.nan])).tolist() == [127] * 3
    assert scale_of(np.array([448.0])) == 1 and scale_of(np.array([449.0])) == 2 and scale_of(np.array([3.5])) == 2 ** -7


@gpu
@pytest.mark.parametrize("ps", [16, 32])
@pytest.mark.parametrize("kind,layout", [("bf16", "rows"), ("bf16", "prompt"), ("f16", "part"), ("f32", "prompt"),
                                         ("f32", "part")])
def test_rows_are_stored_and_read_back(ps, kind, layout):
    _need_gpu()
    s = Store(2, 3, ps, 5, 5, seed=ps)
    for count in ([1, 0, 15, 16, 17], [40, 3, 1, 0, 33], [0, 0, 0, 0, 0], [1, 1, 1, 1, 1], [20, 60, 2, 31, 16]):
        k, v = s.rows(sum(count) + 2, kind, layout=layout)        # two rows too many: not read
        s.write(k, v, count)
        s.check()
    T = sum(s.n)
    k, v = (torch.full((T + 1, 2, 3, D), 7.0, dtype=TYPES[kind], device="cuda") for _ in range(2))
    md.md_read_cache8(k, v, s.pool, s.sc, s.bt, np.zeros(5, np.int32), np.array(s.n, np.int32))
    want = np.zeros((2, T, 2, 3, D))
    row = 0
    for b in range(5):
        for t in range(s.n[b]):
            phys, slot = s.table[b, t // ps], t % ps
            x = decode(s.codes[:, phys, :, :, slot]) * s.scales[:, phys, :, :, slot // BLOCK][..., None]
            want[:, row] = np.moveaxis(x, 2, 0)
            row += 1
    for got, w in ((k, want[0]), (v, want[1])):
        assert torch.equal(got[:T].cpu(), torch.from_numpy(w).to(TYPES[kind])) and (got[T] == 7).all()
    s.check()                                                     # a read writes nothing
    # a part of each sequence, into rows that lie as a cache takes them
    first = np.array([n // 3 for n in s.n], np.int32)
    count = np.array([n - n // 3 - n // 5 for n in s.n], np.int32)
    part = torch.full((2, 3, int(count.sum()), D), 7.0, dtype=TYPES[kind], device="cuda").permute(2, 0, 1, 3)
    other = torch.empty_like(part)
    md.md_read_cache8(part, other, s.pool, s.sc, s.bt, first, count)
    at = np.concatenate([np.arange(f, f + c) + sum(s.n[:b]) for b, (f, c) in enumerate(zip(first, count))])
    assert torch.equal(part, k[torch.from_numpy(at).cuda()]) and torch.equal(other, v[torch.from_numpy(at).cuda()])


@gpu
@pytest.mark.parametrize("batch", [16, 17, md.MD_MAX_BATCH])
def test_batches_up_to_the_largest(batch):
    """Sequences without new tokens among them."""
    _need_gpu()
    s = Store(1, 1, 16, batch, 2, seed=batch)
    for step in range(2):
        count = [(b * 7 + step) % 13 for b in range(batch)]
        k, v = s.rows(sum(count), "bf16")
        s.write(k, v, count)
    s.check()
    k, v = (torch.zeros((sum(s.n), 1, 1, D), device="cuda") for _ in range(2))
    md.md_read_cache8(k, v, s.pool, s.sc, s.bt, np.zeros(batch, np.int32), np.array(s.n, np.int32))
    at = [(s.table[b, t // 16], t % 16) for b in range(batch) for t in range(s.n[b])]
    for x, which in ((k, 0), (v, 1)):
        want = np.stack([decode(s.codes[0, p, 0, which, t]) * s.scales[0, p, 0, which, 0] for p, t in at])
        assert np.array_equal(x[:, 0, 0].cpu().numpy(), want.astype(np.float32))


@gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_scales_of_blocks_grow_with_their_tokens(kind):
    """Token by token, each larger or smaller than those before by up to 2^20: codes move to the new
    scale, the small ones into the subnormal range and to zero."""
    _need_gpu()
    s = Store(1, 2, 16, 3, 3, seed=5)
    for step in range(36):
        size = 2.0 ** s.rng.integers(-12, 7)
        k, v = s.rows(3, kind, size)
        if step % 5 == 0:
            k.zero_()
        s.write(k, v, [1, 1 if step % 2 else 0, 1] if step % 2 else [1, 0, 1])
        s.check()


@gpu
def test_values_at_the_ends_of_the_ranges():
    """The largest and smallest fp32 values, exactly 448 and 449 scales, zeros of both signs; what is
    not finite becomes NaN and does not change its block's scale."""
    _need_gpu()
    s = Store(1, 1, 16, 6, 1, seed=8)
    x = np.zeros((6, 16, 1, 1, D))
    x[0, :] = s.rng.standard_normal((16, 1, 1, D)) * 3e38
    x[1, :] = s.rng.standard_normal((16, 1, 1, D)) * 1e-38
    x[2, :] = s.rng.standard_normal((16, 1, 1, D)) * 1e-44
    x[3, 0, 0, 0, :4] = [448, -448, 0.0, -0.0]
    x[4, 0, 0, 0, :3] = [448.0001, 1, -1]
    x[5] = s.rng.standard_normal((16, 1, 1, D))
    x[5, 3, 0, 0, :3] = [math.inf, -math.inf, math.nan]
    with np.errstate(over="ignore"):
        rows = torch.from_numpy(np.clip(x, -3.4e38, 3.4e38).astype(np.float32)).flatten(0, 1).cuda()
    bad = torch.from_numpy(x[5, 3, 0, 0, :3]).float().cuda()
    rows[5 * 16 + 3, 0, 0, :3] = bad
    s.write(rows, rows.clone(), [16] * 6)
    s.check()
    assert s.scales[0, s.table[5, 0], 0, 0, 0] < 1 and (s.codes[0, s.table[5, 0], 0, 0, 3, :3] & 127 == 127).all()


@gpu
def test_pages_outside_the_pool():
    _need_gpu()
    s = Store(1, 2, 32, 2, 3, seed=9)
    s.table[0, 1], s.table[1, 0], s.table[1, 2] = -1, s.P, 1 << 30
    s.to_gpu()
    k, v = s.rows(150, "bf16")
    s.write(k, v, [80, 70])
    s.check()
    md.md_read_cache8(k, v, s.pool, s.sc, s.bt, [0, 0], [80, 70])
    nan = torch.isnan(k).flatten(1).all(1).cpu().numpy()
    assert nan.tolist() == [32 <= t < 64 for t in range(80)] + [t < 32 or t >= 64 for t in range(70)]


@gpu
def test_offsets_beyond_32_bits():
    """The last pages of a pool of 5 GB, and of rows of more than 2^31 elements apart."""
    _need_gpu()
    P, L = 160000, 4
    pool = torch.zeros((L, P, 2, 2, 16, D), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((L, P, 2, 2, 1), device="cuda")
    table = torch.tensor([[P - 1, 3, P - 2]], dtype=torch.int32, device="cuda")
    wide = torch.empty((L, 2, 48 + (1 << 20), D), dtype=torch.bfloat16, device="cuda")
    k = wide.permute(2, 0, 1, 3)[-48:]
    k.normal_()
    v = torch.randn((48, L, 2, D), device="cuda").bfloat16()
    md.md_write_cache8(k, v, pool, scales, table, [0], [48])
    a, b = torch.empty_like(v), torch.empty_like(v)
    md.md_read_cache8(a, b, pool, scales, table, [0], [48])
    for x, y, which in ((k, a, 0), (v, b, 1)):
        blocks = x.float().reshape(3, 16, L, 2, D)
        s = torch.stack([scales[:, p, :, which, 0] for p in (P - 1, 3, P - 2)])       # [3][L][2]
        want = (blocks / s[:, None, :, :, None]).to(torch.float8_e4m3fn).float() * s[:, None, :, :, None]
        assert torch.equal(y.float(), want.reshape(48, L, 2, D))
    assert int((scales != 0).sum()) == 3 * L * 4
    used = torch.zeros(P, dtype=torch.bool, device="cuda")
    used[[P - 1, 3, P - 2]] = True
    assert not pool[:, ~used][:, ::997].any()


@gpu
def test_on_another_stream_and_in_a_graph():
    _need_gpu()
    s = Store(2, 2, 16, 3, 4, seed=11)
    side = torch.cuda.Stream()
    k, v = s.rows(60, "bf16")
    side.wait_stream(torch.cuda.current_stream())
    s.write(k, v, [20, 33, 7], stream=side)
    side.synchronize()
    s.check()
    k, v = s.rows(3, "f32")
    out = [torch.zeros_like(k), torch.zeros_like(v)]
    first = np.array(s.n, np.int32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        md.md_write_cache8(k, v, s.pool, s.sc, s.bt, first, [1, 1, 1])
        md.md_read_cache8(out[0], out[1], s.pool, s.sc, s.bt, first, [1, 1, 1])
    s.check()                                                     # captured, not run
    for _ in range(3):                                            # the same slots again, with other rows
        k.normal_()
        v.normal_()
        graph.replay()
        write_ref(s.codes, s.scales, k.double().cpu().numpy(), v.double().cpu().numpy(), s.table, first, [1, 1, 1])
        s.check()
        for x, which in ((out[0], 0), (out[1], 1)):
            for b in range(3):
                phys, slot = s.table[b, s.n[b] // 16], s.n[b] % 16
                want = decode(s.codes[:, phys, :, which, slot]) * s.scales[:, phys, :, which, 0][..., None]
                assert np.array_equal(x[b].cpu().numpy(), want.astype(np.float32))


# ------------------------------------------------------------- refusals, on the CPU ----
def _args(**kw):
    a = md.md_cache8_args()
    first, count = np.array([3, 0], np.int32), np.array([20, 5], np.int32)
    d = dict(batch=2, num_layers=2, num_kv_heads=2, page_size=16, max_pages_per_seq=4, num_phys_pages=9, type=md.MD_TYPE_BF16,
             first_host=first.ctypes.data, count_host=count.ctypes.data, k=1 << 20, v=1 << 20, k_row=512, k_layer=256,
             k_head=128, v_row=512, v_layer=256, v_head=128, pool_dev=1 << 20, scales_dev=1 << 20,
             block_table_dev=1 << 20, stream=None)
    hold = [first, count]
    for n, x in kw.items():
        if isinstance(x, list):
            x = np.array(x, np.int32)
            hold.append(x)
            x = x.ctypes.data
        d[n] = x
    for n, x in d.items():
        setattr(a, n, x)
    a.hold = hold
    return a


REFUSED = [dict(batch=0), dict(batch=257), dict(num_layers=0), dict(num_layers=256), dict(num_kv_heads=0),
           dict(page_size=8), dict(page_size=64), dict(max_pages_per_seq=1), dict(max_pages_per_seq=1 << 15),
           dict(num_phys_pages=0), dict(num_phys_pages=1 << 27), dict(type=md.MD_TYPE_E4M3), dict(type=-1),
           dict(first_host=None), dict(count_host=None), dict(first_host=[-1, 0]), dict(count_host=[-1, 3]),
           dict(first_host=[60, 0]), dict(first_host=[(1 << 31) - 1, 0], count_host=[(1 << 31) - 1, 0]), dict(k=None),
           dict(v=None), dict(k=(1 << 20) + 4), dict(type=md.MD_TYPE_F32, v=(1 << 20) + 8), dict(k_row=6), dict(v_head=-2),
           dict(pool_dev=None), dict(pool_dev=(1 << 20) + 8), dict(scales_dev=None), dict(scales_dev=(1 << 20) + 2),
           dict(block_table_dev=None), dict(block_table_dev=(1 << 20) + 2)]


@pytest.mark.parametrize("call", ["md_write_cache8", "md_read_cache8"])
@pytest.mark.parametrize("bad", REFUSED, ids=[",".join(x) + str(i) for i, x in enumerate(REFUSED)])
def test_arguments_are_refused_before_any_launch(call, bad):
    a = _args(**bad)
    assert getattr(md.lib(), call)(ctypes.byref(a)) == md.MD_ERR_INVALID_ARG
    assert getattr(md.lib(), call)(None) == md.MD_ERR_INVALID_ARG


@pytest.mark.parametrize("call", ["md_write_cache8", "md_read_cache8"])
def test_a_call_of_no_tokens_is_done(call):
    a = _args(count_host=[0, 0], k=None, v=None)
    assert getattr(md.lib(), call)(ctypes.byref(a)) == md.MD_OK
