"""Rows of md_attend_cache whose copies do not land in time: they are NaN, the others are not touched by it, the
launch ends, and the next one works.  The kernel's source is built once more with an entry that sets the limit
of the waits, and a step that each warp takes for a lost one."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2607_10582_gb300 as md
from paper_2607_10582_gb300 import build as mdbuild
from tests.attend_forms import FORMS
from tests.test_attend_cache import Case, _need_gpu

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def give_up(tmp_path_factory):
    _need_gpu()
    mdbuild.build()
    objs = [os.path.join(mdbuild.OBJ_DIR, s + ".o") for s in mdbuild.SOURCES if s != "md_attend.cu"]
    if not all(map(os.path.exists, objs)):
        mdbuild.build(force=True)
    lib = str(tmp_path_factory.mktemp("give_up") / "libgiveup.so")
    r = subprocess.run(["nvcc", *mdbuild.ARCH, *mdbuild.FLAGS, "-shared", "-o", lib, os.path.join(ROOT, "tests", "c", "attend_give_up.cu"),
                        *objs, "-cudart", "static"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    f = ctypes.CDLL(lib).attend_give_up
    f.argtypes, f.restype = [ctypes.POINTER(md.md_attend_cache_args), ctypes.c_longlong, ctypes.c_int], ctypes.c_int

    def call(c, workspace, limit_ns, lost_step):
        out = torch.full_like(c.q, 7.0)
        lse = torch.full((c.B, c.L, c.Hq), 7.0, device="cuda")
        ws = torch.full((md.MD_ATTEND_WORKSPACE,), 255, dtype=torch.uint8, device="cuda") if workspace else None
        a = md.md_attend_cache_args(c.B, c.L, c.Hq, c.Hkv, c.ps, c.W, c.P, md.MD_TYPE_BF16 if c.scales is None else md.MD_TYPE_E4M3,
                                    -1, 0, c.q.data_ptr(), c.pool.data_ptr(), c.scales.data_ptr() if c.scales is not None else None,
                                    c.bt.data_ptr(), c.n.ctypes.data, out.data_ptr(), lse.data_ptr(), ws.data_ptr() if workspace else None,
                                    ws.numel() if workspace else 0, torch.cuda.current_stream().cuda_stream)
        assert f(ctypes.byref(a), limit_ns, lost_step) == md.MD_OK
        torch.cuda.synchronize()
        return out, lse

    return call


def _gone(c, got, want):
    """Which (sequence, layer, KV head) rows gave up: all of their heads are NaN, and all else is as it should be."""
    shape = (c.B, c.L, c.Hkv, -1)
    nan = got[0].isnan().view(shape).all(-1)
    assert torch.equal(nan, got[0].isnan().view(shape).any(-1))
    assert torch.equal(got[1].isnan().view(shape), nan[..., None].expand(-1, -1, -1, c.G))
    for x, y in zip(got, want):
        keep = ~nan[..., None].expand(-1, -1, -1, x.view(shape).shape[-1])
        assert torch.equal(x.view(shape)[keep], y.view(shape)[keep])
    return nan


@gpu
@pytest.mark.parametrize("kind,L,Hkv,workspace,lengths,form", FORMS)
def test_a_row_that_gives_up(give_up, kind, L, Hkv, workspace, lengths, form):
    c = Case(kind, L, 3 * Hkv, Hkv, 16, lengths, seed=sum(lengths))
    want = c.attend(bool(workspace))
    step = 32 if kind == "e4m3" else 16
    warps = max(form[0], 1) * (form[1] if form[0] else 1)         # of a row that is not split
    for lost in (0, 1, 2, 5):
        gone = _gone(c, give_up(c, workspace, 2 * 10 ** 9, lost), want)
        if lost == 0 or not form[2]:
            rounds = torch.from_numpy(np.array([-(-(-(-n // step)) // warps) for n in lengths])).cuda()
            assert torch.equal(gone, (rounds > lost)[:, None, None].expand_as(gone)), lost
    again = give_up(c, workspace, 2 * 10 ** 9, -1)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])


@gpu
@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_a_limit_shorter_than_a_copy(give_up, kind):
    """What was in flight lands before a launch ends, whichever rows gave up: the next call is right."""
    for lengths, workspace in (([700] * 40, False), ([20000, 3000, 0, 64], False), ([90000], True), ([60] * 200, False)):
        c = Case(kind, 1, 8, 2, 16, lengths, seed=7)
        want = c.attend(workspace)
        for _ in range(20):
            _gone(c, give_up(c, workspace, 0, -1), want)
            again = c.attend(workspace)
            assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
