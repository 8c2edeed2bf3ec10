"""What the Python side of the row and page calls lets through, with stand-ins for device
tensors and for the library: no GPU."""
import contextlib
import math
import sys
import types

import numpy as np
import pytest

import paper_2607_10582_gb300 as md

torch = pytest.importorskip("torch")
D = 128


class Stub:
    """What the checks read of a device tensor."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=0):
        self.t = torch.empty(shape, dtype=dtype, device="meta")
        self.shape, self.dtype, self.device, self.is_cuda = self.t.shape, dtype, torch.device("cuda", device), True
        self.dim, self.stride, self.numel = self.t.dim, self.t.stride, self.t.numel
        self.element_size, self.is_contiguous = self.t.element_size, self.t.is_contiguous

    def data_ptr(self):
        return 1 << 20


class Library:
    """Records the calls that would be launched."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or md.MD_OK


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(md, "lib", lambda: lib)
    monkeypatch.setattr(md, "_torch_calls", md._NoCalls)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=0))
    return lib


def _rows(**kw):
    i32, f32 = torch.int32, torch.float32
    a = dict(q=Stub(4, 3, D), k=Stub(4, 2, D), v=Stub(4, 2, D), q_out=Stub(4, 3, D), k_out=Stub(4, 2, D), v_out=Stub(4, 2, D),
             positions=Stub(4, dtype=i32), table=Stub(9, 64, 2, dtype=f32), q_weight=Stub(D, dtype=f32),
             k_weight=Stub(D, dtype=f32))
    a.update(kw)
    rows = [a.pop(n) for n in ("q", "k", "v", "q_out", "k_out", "v_out")]
    md.md_norm_rope(*rows, **a)


@pytest.mark.parametrize("value", [False, 0, None, np.False_, True, 1, np.True_])
def test_interleaved_is_taken_for_its_truth(library, value):
    _rows(interleaved=value)
    assert library.calls[0][1][0]._obj.interleaved == (1 if value else 0)


@pytest.mark.parametrize("name", ["q_out", "k_out", "v_out"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32, torch.int32, torch.uint8])
def test_rows_are_written_as_bf16_only(library, name, dtype):
    """An f16 tensor would receive bf16 bits."""
    with pytest.raises(md.MemDecayError):
        _rows(**{name: Stub(4, 3 if name == "q_out" else 2, D, dtype=dtype)})
    assert not library.calls


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int16, torch.uint16])
def test_rows_are_written_as_bf16_or_its_bits(library, dtype):
    f16 = torch.float16
    _rows(q=Stub(4, 3, D, dtype=f16), k=Stub(4, 2, D, dtype=f16), v=Stub(4, 2, D, dtype=f16),
          **{n: Stub(4, 3 if n == "q_out" else 2, D, dtype=dtype) for n in ("q_out", "k_out", "v_out")})
    assert [c[0] for c in library.calls] == ["md_norm_rope"]


def _pages(call, **kw):
    """A call of one sequence, 2 layers, 4 pages of 16 tokens, 2 KV heads and 8 query heads."""
    i32, f32 = torch.int32, torch.float32
    a = dict(q=Stub(1, 2, 8, D), pool=Stub(2, 4, 2, 2, 16, D), bounds=Stub(2, 4, 2, 2, D), block_table=Stub(1, 4, dtype=i32),
             scores=Stub(1, 2, 2, 4, dtype=f32), page_ids=Stub(1, 2, 2, 3, dtype=i32), out=Stub(1, 2, 8, D),
             mass=Stub(1, 2, 2, 48, dtype=f32), n_tokens=[50])
    a.update(kw)
    names, keywords = CALLS[call]
    getattr(md, call)(*(a[n] for n in names), **{n: a[n] if n in a else 16 for n in keywords})


CALLS = {
    "md_page_bounds": (("pool", "block_table", "n_tokens", "bounds"), ()),
    "md_page_scores": (("q", "bounds", "block_table", "n_tokens", "scores"), ("page_size",)),
    "md_page_top": (("scores", "n_tokens", "page_ids"), ("page_size",)),
    "md_attend_pages": (("q", "pool", "block_table", "n_tokens", "page_ids", "out"), ("mass",)),
}
TENSORS = [(c, n) for c, (names, keywords) in CALLS.items() for n in names + keywords if n not in ("n_tokens", "page_size")]


def _elsewhere(t):
    return Stub(*t.shape, dtype=t.dtype, device=1)


@pytest.mark.parametrize("call,name", TENSORS)
def test_page_calls_take_tensors_of_one_device(library, call, name):
    _pages(call)
    assert [c[0] for c in library.calls] == [call]
    like = dict(q=Stub(1, 2, 8, D), pool=Stub(2, 4, 2, 2, 16, D), bounds=Stub(2, 4, 2, 2, D),
                block_table=Stub(1, 4, dtype=torch.int32), scores=Stub(1, 2, 2, 4, dtype=torch.float32),
                page_ids=Stub(1, 2, 2, 3, dtype=torch.int32), out=Stub(1, 2, 8, D),
                mass=Stub(1, 2, 2, 48, dtype=torch.float32))[name]
    with pytest.raises(md.MemDecayError) as e:
        _pages(call, **{name: _elsewhere(like)})
    assert e.value.status == md.MD_ERR_INVALID_ARG and len(library.calls) == 1


@pytest.mark.parametrize("name", ["q", "k", "v", "q_out", "k_out", "v_out", "positions", "table", "q_weight", "k_weight"])
def test_rows_take_tensors_of_one_device(library, name):
    shape = dict(positions=(4,), table=(9, 64, 2), q_weight=(D,), k_weight=(D,), q=(4, 3, D), q_out=(4, 3, D))
    dtype = dict(positions=torch.int32, table=torch.float32, q_weight=torch.float32, k_weight=torch.float32)
    with pytest.raises(md.MemDecayError) as e:
        _rows(**{name: Stub(*shape.get(name, (4, 2, D)), dtype=dtype.get(name, torch.bfloat16), device=1)})
    assert e.value.status == md.MD_ERR_INVALID_ARG and not library.calls


@pytest.mark.parametrize("call,name", [x for x in TENSORS if x[1] != "mass"])
def test_page_calls_say_which_tensor_is_missing(library, call, name):
    with pytest.raises(md.MemDecayError) as e:
        _pages(call, **{name: None})
    assert e.value.status == md.MD_ERR_INVALID_ARG and name in str(e.value) and not library.calls


def test_a_rotation_needs_positions(library):
    with pytest.raises(md.MemDecayError) as e:
        _rows(positions=None)
    assert e.value.status == md.MD_ERR_INVALID_ARG and "positions" in str(e.value) and not library.calls
    _rows(positions=None, table=None)
    assert len(library.calls) == 1


@pytest.mark.parametrize("counts", [np.array([(1 << 32) + 50]), np.array([50.5]), [50.5], np.array([math.nan]), [1 << 70]])
@pytest.mark.parametrize("call", list(CALLS))
def test_token_counts_are_taken_as_they_are(library, call, counts):
    """A count that int32 does not hold is refused, not wrapped or cut."""
    with pytest.raises(md.MemDecayError):
        _pages(call, n_tokens=counts)
    assert not library.calls


@pytest.mark.parametrize("counts", [[50], (50,), np.array([50]), np.array([50, 9], np.int16), np.array([50.0]),
                                    torch.tensor([50])])
def test_token_counts_of_other_types_are_converted(library, counts):
    _pages("md_page_top", n_tokens=counts)
    assert len(library.calls) == 1


@pytest.mark.parametrize("axes", [np.full(64, 256), np.full(64, -256), [0.5] * 64])
def test_axes_are_taken_as_they_are(library, axes):
    with pytest.raises(md.MemDecayError):
        _rows(positions=Stub(2, 4, dtype=torch.int32), axes=axes)
    assert not library.calls
    _rows(positions=Stub(2, 4, dtype=torch.int32), axes=[0, 1] * 32)
    assert len(library.calls) == 1


class Streams:
    """Stands in for torch: which stream is current when memory is taken, and what is ordered
    behind what."""

    uint8, float32 = torch.uint8, torch.float32

    def __init__(self):
        self.log, self.now, self.cuda = [], "current", self

    @contextlib.contextmanager
    def stream(self, s):
        was, self.now = self.now, s
        yield
        self.now = was

    def current_stream(self, *a):
        return self.now

    def current_device(self):
        return 0

    def empty(self, *a, **kw):
        self.log.append(("taken", self.now))
        return types.SimpleNamespace(data_ptr=lambda: 1 << 20, is_cuda=True, device=torch.device("cuda", 0),
                                     record_stream=lambda s: self.log.append(("used", s)))


class Stream:
    cuda_stream = 77

    def __init__(self, torch_):
        self.torch = torch_

    def wait_stream(self, s):
        self.torch.log.append(("waits", s))


def test_sparse_buffer_is_ordered_before_its_first_use(library):
    """The allocator may give out a block that another stream's kernels still write: the handle's
    stream, which uses the buffer, is the one it is taken on."""
    c, t = object.__new__(md.Cache), Streams()
    c.torch, c.stream, c.device, c.h, c.cfg = t, Stream(t), "cuda:0", None, md.md_config()
    library.md_sparse_bytes = lambda *a: 1000
    c.sparse_enable(4)
    assert t.log[0] == ("taken", c.stream) or ("waits", "current") in t.log
    assert library.calls[0][0] == "md_sparse_enable"


def test_table_is_ordered_before_its_first_use(library, monkeypatch):
    """A table written on a given stream: that stream waits for whoever had the memory, and the
    memory is not given out again before that stream is done with it."""
    t = Streams()
    monkeypatch.setitem(sys.modules, "torch", t)
    s = Stream(t)
    md.md_rope_table(np.ones(64), 10, stream=s)
    assert library.calls[0][0] == "md_rope_table" and library.calls[0][1][-1] == 77
    assert ("taken", s) in t.log or (("waits", "current") in t.log and ("used", s) in t.log)


def test_workspace_is_ordered_before_its_first_use(library, monkeypatch):
    """The same for a handle's workspace."""
    t = Streams()
    for name in ("int32", "int64", "int16"):
        setattr(t, name, getattr(torch, name))
    t.device = lambda x: x
    monkeypatch.setitem(sys.modules, "torch", t)
    monkeypatch.setattr(md, "_fast", md._NoCalls)
    library.md_workspace_size = lambda *a: 1000
    s = Stream(t)
    c = md.Cache(1, 1, 1, 16, 1, 4, 4, stream=s, device="cuda:0")
    assert t.log[0] == ("taken", s) or ("waits", "current") in t.log
    assert library.calls[0][0] == "md_create"
    c.h = None
