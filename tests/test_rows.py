"""md_norm_rope and md_rope_table against the formulas in 64 bits, and their refusals.

Tolerance of a row element: the output's rounding to bf16 (half an ulp, at most 2^-8 of the
value) and what 32-bit arithmetic adds before it: the sum of 128 squares, its root and the
table entry come to a few 2^-24 each, so 2^-18 of the two channels that a rotation mixes is
ample (about 60 roundings)."""
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


def _need_gpu():
    if not torch.cuda.is_available():  # pragma: no cover
        pytest.skip("needs a CUDA GPU")


def _freq(pairs):
    return np.exp(np.arange(pairs) * (-math.log(1e6) / max(1, pairs)))


def _ref(x, weight, eps, pos, freq, axes, interleaved):
    """float64 [T][H][128] -> (result, bound of what 32-bit arithmetic mixes)."""
    y = x
    if weight is not None:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    out, size = y.copy(), np.abs(y)
    n = len(freq)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        angle = (pos[axes[i]].astype(np.float64) * freq[i])[:, None]
        c, s = np.cos(angle), np.sin(angle)
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size


def _check(got, ref, size):
    got = got.double().cpu().numpy()
    far = np.abs(got - ref) - (2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * size + 1e-38)
    assert got.shape == ref.shape and np.nanmax(far, initial=-1.0) <= 0 and not np.isnan(got).any()


@gpu
@pytest.mark.parametrize("T,Hq,Hkv,dtype,R,inter,axes,norm", [
    (1, 12, 2, "bfloat16", 128, False, 1, True),
    (1, 1, 1, "float32", 128, True, 1, True),
    (7, 16, 2, "float16", 64, False, 3, True),
    (33, 3, 1, "bfloat16", 8, False, 1, False),
    (65, 8, 4, "float32", 40, True, 2, True),
    (129, 28, 4, "bfloat16", 128, True, 4, False),
    (1000, 16, 2, "bfloat16", 96, False, 3, True),
    (2049, 12, 2, "float16", 128, False, 1, True),
    (5, 2, 1, "bfloat16", 0, False, 1, True),
    (70001, 1, 1, "bfloat16", 128, False, 1, True),
])
def test_rows_follow_the_formula(T, Hq, Hkv, dtype, R, inter, axes, norm):
    _need_gpu()
    g = torch.Generator(device="cuda").manual_seed(T + R)
    rng = np.random.default_rng(T)
    rows = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device="cuda").to(getattr(torch, dtype))
    rows[T // 2, 0] *= 1e-3                       # a row whose eps matters
    qw, kw = (1 + 0.3 * torch.randn((2, D), generator=g, device="cuda")).unbind(0) if norm else (None, None)
    n = R // 2
    freq = _freq(n)
    table = md.md_rope_table(freq, 4099) if R else None
    pos = rng.integers(0, 4099, (axes, T)).astype(np.int32)
    pos[0, 0], pos[0, -1] = 0, 4098
    which = rng.integers(0, axes, n).astype(np.uint8)
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    q_out = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
    k_out, v_out = (torch.empty((Hkv, T, D), dtype=torch.bfloat16, device="cuda").transpose(0, 1) for _ in range(2))
    p = torch.from_numpy(pos).cuda()
    md.md_norm_rope(q, k, v, q_out, k_out, v_out, positions=p if axes > 1 else p[0], table=table, q_weight=qw,
                    k_weight=kw, eps=1e-5, axes=which if axes > 1 else None, interleaved=inter)
    for x, w, y in ((q, qw, q_out), (k, kw, k_out)):
        ref, size = _ref(x.double().cpu().numpy(), None if w is None else w.double().cpu().numpy(), 1e-5, pos, freq,
                         which if axes > 1 else np.zeros(n, int), inter)
        _check(y, ref, size)
    assert torch.equal(v_out, v.to(torch.bfloat16))


@gpu
def test_table_is_rounded_once_from_64_bits():
    _need_gpu()
    freq = _freq(64)
    t = md.md_rope_table(freq, 262144, scale=0.75).double().cpu().numpy()
    at = np.array([0, 1, 2, 777, 131071, 262143])
    angle = at[:, None] * freq
    for i, f in ((0, np.cos), (1, np.sin)):
        x = 0.75 * f(angle)
        half_ulp = np.spacing(np.abs(x).astype(np.float32)).astype(np.float64) / 2
        assert (np.abs(t[at, :, i] - x) <= half_ulp + 1e-10).all()      # the angle itself: 2^-53 of 262143


@gpu
def test_parts_of_a_step_and_in_place():
    """Outputs as one layer's part of a step's tensors; queries alone, keys alone; a row
    rotated where it is; what lies between the rows stays."""
    _need_gpu()
    T, L, Hq, Hkv = 9, 3, 4, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn((T, Hq, D), generator=g, device="cuda").bfloat16()
    k = torch.randn((T, Hkv, D), generator=g, device="cuda").bfloat16()
    table = md.md_rope_table(_freq(64), 64)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    step_q = torch.zeros((T, L, Hq, D), dtype=torch.bfloat16, device="cuda")
    step_k = torch.zeros((T, L, Hkv, D), dtype=torch.bfloat16, device="cuda")
    md.md_norm_rope(q, None, None, step_q[:, 1], None, None, positions=pos, table=table)
    md.md_norm_rope(None, k, None, None, step_k[:, 2], None, positions=pos, table=table)
    both_q, both_k = torch.empty_like(q), torch.empty_like(k)
    md.md_norm_rope(q, k, None, both_q, both_k, None, positions=pos, table=table)
    assert torch.equal(step_q[:, 1], both_q) and torch.equal(step_k[:, 2], both_k)
    assert not step_q[:, ::2].any() and not step_k[:, :2].any()
    md.md_norm_rope(q, k, None, q, k, None, positions=pos, table=table)
    assert torch.equal(q, both_q) and torch.equal(k, both_k)


@gpu
def test_infinities_and_positions_outside_the_table():
    _need_gpu()
    x = torch.randn((4, 2, D), device="cuda").bfloat16()
    x[1, 0, 5] = math.nan
    y = torch.empty_like(x)
    table = md.md_rope_table(_freq(32), 10)                 # channels 64.. are not rotated
    pos = torch.tensor([3, 3, -1, 10], dtype=torch.int32, device="cuda")
    md.md_norm_rope(x, None, None, y, None, None, positions=pos, table=table)
    nan = y.isnan().cpu()
    assert nan[2:, :, :64].all() and not nan[2:, :, 64:].any()
    assert nan[1, 0].nonzero().flatten().tolist() == [5, 37] and not nan[0].any() and not nan[1, 1].any()
    assert torch.equal(y[2:, :, 64:], x[2:, :, 64:])


@gpu
def test_no_tokens_and_no_rotation():
    _need_gpu()
    x, y = (torch.ones((0, 4, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = md.md_rope_table(_freq(64), 8)
    md.md_norm_rope(x, None, None, y, None, None, positions=torch.zeros(0, dtype=torch.int32, device="cuda"), table=table)
    x = torch.randn((6, 4, D), device="cuda")
    y = torch.empty((6, 4, D), dtype=torch.bfloat16, device="cuda")
    md.md_norm_rope(x, None, None, y, None, None, positions=None, table=None)        # a rounding copy
    assert torch.equal(y, x.bfloat16())


@gpu
def test_unaligned_rows():
    """Rows at 8-byte addresses and odd multiples of 4 elements apart, and rotary_dim = 8 mod 16,
    take another kernel: the same values."""
    _need_gpu()
    T, H = 37, 5
    g = torch.Generator(device="cuda").manual_seed(8)
    big = torch.randn((T, H * 132 + 4), generator=g, device="cuda").bfloat16()
    off = big[:, 4:].view(T, H * 132)[:, :H * 132].unflatten(1, (H, 132))[..., :D]    # head stride 132, base + 8 bytes
    even = off.contiguous()
    table, w = md.md_rope_table(_freq(64), 99), 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    pos = torch.randint(0, 99, (2, T), generator=g, device="cuda", dtype=torch.int32)
    axes = np.arange(64, dtype=np.uint8) % 2
    for inter in (False, True):
        for weight in (None, w):
            a, b = (torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            md.md_norm_rope(off, None, None, a, None, None, positions=pos, table=table, q_weight=weight, axes=axes,
                            interleaved=inter)
            md.md_norm_rope(even, None, None, b, None, None, positions=pos, table=table, q_weight=weight, axes=axes,
                            interleaved=inter)
            for y in (a, b):
                ref, size = _ref(even.double().cpu().numpy(), None if weight is None else w.double().cpu().numpy(), 1e-6,
                                 pos.cpu().numpy(), _freq(64), axes, inter)
                _check(y, ref, size)


@gpu
def test_calls_without_the_c_module_are_the_same(monkeypatch):
    """Where Python's headers are missing every call goes through ctypes."""
    _need_gpu()
    x = torch.randn((40, 10, D), device="cuda").half()
    table, pos = md.md_rope_table(_freq(64), 4000), torch.randint(0, 4000, (3, 40), dtype=torch.int32, device="cuda")
    w, axes = torch.rand(D, device="cuda"), np.arange(64, dtype=np.uint8) % 3
    outs = []
    for b in (md._binding(), md._NoCalls):
        monkeypatch.setattr(md, "_torch_calls", None)
        monkeypatch.setattr(md, "_fast", b)
        y = torch.zeros((40, 10, D), dtype=torch.bfloat16, device="cuda")
        md.md_norm_rope(x[:, :6], x[:, 6:8], x[:, 8:], y[:, :6], y[:, 6:8], y[:, 8:], positions=pos, table=table,
                        q_weight=w, axes=axes, interleaved=True)
        outs.append(y)
    assert torch.equal(*outs) and outs[0].any()


@gpu
@pytest.mark.parametrize("value", [False, 0, None, np.False_, True, 1, np.True_])
def test_interleaved_is_taken_for_its_truth(value, monkeypatch):
    _need_gpu()
    x = torch.randn((5, 4, D), device="cuda").bfloat16()
    table, pos = md.md_rope_table(_freq(64), 50), torch.arange(5, dtype=torch.int32, device="cuda")
    want = torch.empty_like(x)
    md.md_norm_rope(x, None, None, want, None, None, positions=pos, table=table, interleaved=True if value else False)
    for b in (md._binding(), md._NoCalls):
        monkeypatch.setattr(md, "_torch_calls", None)
        monkeypatch.setattr(md, "_fast", b)
        got = torch.zeros_like(x)
        md.md_norm_rope(x, None, None, got, None, None, positions=pos, table=table, interleaved=value)
        assert torch.equal(got, want)


@gpu
def test_rows_on_another_stream():
    """The call goes to the stream it is given, behind the work that stream holds."""
    _need_gpu()
    s = torch.cuda.Stream()
    x = torch.randn((3000, 16, D), device="cuda").bfloat16()
    want, got = torch.empty_like(x), torch.empty_like(x)
    table, pos = md.md_rope_table(_freq(64), 4000), torch.arange(3000, dtype=torch.int32, device="cuda")
    md.md_norm_rope(x, None, None, want, None, None, positions=pos, table=table)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        late = torch.zeros_like(x)
        for _ in range(20):
            late.copy_(x)
        md.md_norm_rope(late, None, None, got, None, None, positions=pos, table=table)
    s.synchronize()
    assert torch.equal(got, want)


@gpu
def test_table_on_another_stream_with_work_pending():
    """Writes that the current stream still has to a block it gave up come before the table's."""
    _need_gpu()
    freq, s = _freq(64), torch.cuda.Stream()
    want = md.md_rope_table(freq, 5000)
    old = torch.empty_like(want)
    big = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for _ in range(100):
        big.fill_(1)                               # some ms
    old.fill_(7.0)
    del old
    got = md.md_rope_table(freq, 5000, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def _args(**kw):
    a = md.md_norm_rope_args()
    base = dict(n_tokens=4, num_q_heads=2, num_kv_heads=1, type=0, rotary_dim=128, num_axes=1, table_len=8, eps=1e-6,
                q=4096, k=4096, v=4096, q_out=4096, k_out=4096, v_out=4096, table=4096, positions=4096, q_token=256,
                q_head=128, k_token=128, v_token=128, q_out_token=256, q_out_head=128, k_out_token=128,
                v_out_token=128)
    base.update(kw)
    for n, x in base.items():
        setattr(a, n, x)
    return a


def test_refusals_come_before_any_launch():
    """Addresses here are made up: a call that is not refused would need a GPU."""
    call = md.lib().md_norm_rope
    assert call(None) == md.MD_ERR_INVALID_ARG
    for bad in (dict(n_tokens=-1), dict(type=3), dict(rotary_dim=4), dict(rotary_dim=136), dict(rotary_dim=-8),
                dict(eps=math.nan), dict(eps=-1.0), dict(q=None), dict(k=None), dict(q_out=None), dict(v_out=None),
                dict(q=4100), dict(q_out=4098), dict(q_token=130), dict(k_out_head=2), dict(type=2, q=4104),
                dict(table=None), dict(table=4104), dict(positions=None), dict(num_axes=0), dict(num_axes=5),
                dict(table_len=0), dict(q_weight=4100), dict(num_q_heads=-1), dict(num_kv_heads=1 << 20)):
        assert call(ctypes.byref(_args(**bad))) == md.MD_ERR_INVALID_ARG, bad
    axis = np.full(64, 1, np.uint8)
    assert call(ctypes.byref(_args(axis_host=axis.ctypes.data))) == md.MD_ERR_INVALID_ARG   # axis 1 of 1
    for empty in (dict(n_tokens=0), dict(num_q_heads=0, num_kv_heads=0)):
        assert call(ctypes.byref(_args(**empty))) == md.MD_OK, empty
    t = md.lib().md_rope_table
    f = np.ones(64)
    for bad in ((None, 128, 4, 1.0, 4096), (f.ctypes.data, 12, 4, 1.0, 4096), (f.ctypes.data, 0, 4, 1.0, 4096),
                (f.ctypes.data, 136, 4, 1.0, 4096), (f.ctypes.data, 128, 0, 1.0, 4096), (f.ctypes.data, 128, 4, 1.0, None),
                (f.ctypes.data, 128, 4, 1.0, 4104)):
        assert t(*bad, None) == md.MD_ERR_INVALID_ARG, bad


def test_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros((2, 3, D), dtype=torch.bfloat16)
    for q, k, v, kw in ((None, None, None, {}), (x, None, None, {}), (x[..., :64], None, None, {}),
                        (x, x.float(), None, {}), (x, x, x[:1], {})):
        with pytest.raises(md.MemDecayError):
            md.md_norm_rope(q, k, v, x, x, x, positions=torch.zeros(2, dtype=torch.int32), table=None, **kw)
