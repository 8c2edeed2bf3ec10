"""What the Python side of the calls on an eight-bit cache lets through, with stand-ins for device
tensors and for the library: no GPU."""
import math
import types

import numpy as np
import pytest

import paper_2607_10582_gb300 as md
from tests.test_binding_checks import Library, Stub

torch = pytest.importorskip("torch")
D = 128
E4M3, F32, I32 = torch.float8_e4m3fn, torch.float32, torch.int32


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(md, "lib", lambda: lib)
    monkeypatch.setattr(md, "_torch_calls", md._NoCalls)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=0))
    return lib


SHAPES = {"k": ((7, 2, 3, D), torch.bfloat16), "v": ((7, 2, 3, D), torch.bfloat16), "pool": ((2, 9, 3, 2, 32, D), E4M3),
          "scales": ((2, 9, 3, 2, 2), F32), "block_table": ((2, 4), I32), "q": ((2, 2, 6, D), torch.bfloat16),
          "out": ((2, 2, 6, D), torch.bfloat16), "lse": ((2, 2, 6), F32), "workspace": ((md.MD_ATTEND_WORKSPACE,), torch.uint8)}
CALLS = {"md_write_cache8": ("k", "v", "pool", "scales", "block_table"), "md_read_cache8": ("k", "v", "pool", "scales", "block_table"),
         "md_attend_cache": ("q", "pool", "block_table", "out", "scales", "lse", "workspace")}
OPTIONAL = ("lse", "workspace")


def _stub(name, device=0, **kw):
    shape, dtype = SHAPES[name]
    return Stub(*kw.get("shape", shape), dtype=kw.get("dtype", dtype), device=device)


def _call(call, first=(0, 3), count=(4, 3), n_tokens=(50, 9), window=None, sinks=0, **kw):
    t = {n: kw[n] if n in kw else _stub(n) for n in CALLS[call]}
    if call == "md_attend_cache":
        md.md_attend_cache(t["q"], t["pool"], t["block_table"], n_tokens, t["out"], scales=t["scales"], window=window, sinks=sinks,
                           lse=t["lse"], workspace=t["workspace"])
    else:
        getattr(md, call)(t["k"], t["v"], t["pool"], t["scales"], t["block_table"], first, count)


EACH = [(c, n) for c, names in CALLS.items() for n in names]


@pytest.mark.parametrize("call,name", EACH)
def test_tensors_of_one_device_and_none_missing(library, call, name):
    _call(call)
    assert [c[0] for c in library.calls] == [call]
    with pytest.raises(md.MemDecayError) as e:
        _call(call, **{name: _stub(name, device=1)})
    assert e.value.status == md.MD_ERR_INVALID_ARG
    if name in OPTIONAL:
        _call(call, **{name: None})
        return
    with pytest.raises(md.MemDecayError) as e:
        _call(call, **{name: None})
    assert e.value.status == md.MD_ERR_INVALID_ARG and len(library.calls) == 1


@pytest.mark.parametrize("call,name", [x for x in EACH if x[1] != "workspace"])
def test_shapes_and_types(library, call, name):
    shape, dtype = SHAPES[name]
    for d in range(len(shape)):
        if name in ("block_table", "k", "v", "pool", "q") and d in {"block_table": (1,), "k": (), "v": (), "pool": (1, 4), "q": ()}[name]:
            continue                                  # a size that the other tensors leave open, or that the library refuses
        bad = tuple(x + 1 if i == d else x for i, x in enumerate(shape))
        with pytest.raises(md.MemDecayError):
            _call(call, **{name: _stub(name, shape=bad)})
    for other in (torch.float64, torch.int8, torch.complex64):
        with pytest.raises(md.MemDecayError):
            _call(call, **{name: _stub(name, dtype=other)})
    with pytest.raises(md.MemDecayError):
        _call(call, **{name: _stub(name, shape=shape[:-1])})
    assert not library.calls


@pytest.mark.parametrize("dtype", [E4M3, torch.uint8])
@pytest.mark.parametrize("call", list(CALLS))
def test_a_pool_is_e4m3_or_its_bits(library, call, dtype):
    _call(call, pool=_stub("pool", dtype=dtype))
    assert len(library.calls) == 1
    for other in (torch.float8_e5m2, torch.bfloat16):
        with pytest.raises(md.MemDecayError):
            _call(call, pool=_stub("pool", dtype=other))


def test_without_scales_a_pool_is_bf16(library):
    _call("md_attend_cache", pool=_stub("pool", dtype=torch.bfloat16), scales=None)
    assert library.calls[0][1][0]._obj.type == md.MD_TYPE_BF16
    with pytest.raises(md.MemDecayError):
        _call("md_attend_cache", scales=None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_rows_of_three_types(library, dtype):
    for call in ("md_write_cache8", "md_read_cache8"):
        _call(call, k=_stub("k", dtype=dtype), v=_stub("v", dtype=dtype))
        with pytest.raises(md.MemDecayError):
            _call(call, k=_stub("k", dtype=dtype), v=_stub("v", dtype=torch.float64))
    a = library.calls[0][1][0]._obj
    assert (a.type, a.k_row, a.k_layer, a.k_head) == (md._row_types()[dtype], 2 * 3 * D, 3 * D, D)
    assert (a.batch, a.num_layers, a.num_kv_heads, a.page_size, a.max_pages_per_seq, a.num_phys_pages) == (2, 2, 3, 32, 4, 9)


@pytest.mark.parametrize("call", ["md_write_cache8", "md_read_cache8"])
@pytest.mark.parametrize("count", [(4, 4), (8, 0), (-1, 3), ((1 << 31) - 1, (1 << 31) - 1), (4,), (1 << 40, 0), (0.5, 1),
                                   (math.nan, 1)])
def test_counts_that_the_rows_do_not_hold(library, call, count):
    with pytest.raises(md.MemDecayError):
        _call(call, count=count)
    with pytest.raises(md.MemDecayError):
        _call(call, first=(0,))
    assert not library.calls


def test_rows_that_lie_on_one_another_are_not_written(library):
    k = Stub(7, 2, 3, D)
    k.stride = lambda d: (0, 3 * D, D, 1)[d]
    _call("md_write_cache8", k=k)
    with pytest.raises(md.MemDecayError):
        _call("md_read_cache8", k=k)
    k.stride = lambda d: (6 * D, 3 * D, 2 * D, 2)[d]
    with pytest.raises(md.MemDecayError):
        _call("md_write_cache8", k=k)
    assert len(library.calls) == 1


@pytest.mark.parametrize("name", ["window", "sinks"])
def test_windows_and_sinks_are_taken_as_given(library, name):
    for x in (0, 5, np.int64(7), 1 << 40, 3.0):
        _call("md_attend_cache", **{name: x})
        assert getattr(library.calls[-1][1][0]._obj, name) == min(int(x), (1 << 31) - 1)
    _call("md_attend_cache")
    assert library.calls[-1][1][0]._obj.window == -1
    n = len(library.calls)
    for x in (-1, -5, 0.5, math.nan, "many", 1 << 70, [3, 4]) + ((None,) if name == "sinks" else ()):
        with pytest.raises(md.MemDecayError):
            _call("md_attend_cache", **{name: x})
    assert len(library.calls) == n


@pytest.mark.parametrize("counts", [[50], [50, math.nan], [50, 1 << 40], np.array([50.5, 1])])
def test_token_counts(library, counts):
    with pytest.raises(md.MemDecayError):
        _call("md_attend_cache", n_tokens=counts)
    assert not library.calls


def test_workspaces(library):
    _call("md_attend_cache")
    a = library.calls[0][1][0]._obj
    assert a.workspace_bytes == md.MD_ATTEND_WORKSPACE and a.workspace_dev
    for bad in (_stub("workspace", dtype=torch.int8), _stub("workspace", dtype=F32)):
        with pytest.raises(md.MemDecayError):
            _call("md_attend_cache", workspace=bad)
