"""What md_write_cache8 states about blocks that hold tokens already, and the reference encoder of its tests."""
import numpy as np
import pytest

import paper_2607_10582_gb300 as md
from tests.test_cache8 import D, Store, _need_gpu, decode, encode

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu


def test_the_reference_rounds_general_values_as_torch_does():
    """Against another implementation of the format, value for value, on inputs that 32 bits hold:
    ordinary ones, subnormal ones, those that become zero, and the largest."""
    r = np.random.default_rng(0)
    for size in (60.0, 1.0, 2.0 ** -6, 2.0 ** -9, 2.0 ** -12):
        x = torch.from_numpy(r.standard_normal(20000) * size).clamp(-448, 448).float()
        want = x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        assert np.array_equal(encode(x.double().numpy()), want), size
    assert encode(np.array([448.0, -448.0, 0.0, -0.0])).tolist() == [126, 254, 0, 128]


@gpu
@pytest.mark.parametrize("ps", [16, 32])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_a_sequence_is_cut_and_goes_on(ps, kind):
    """Cut in the middle of a block, at its start and its end, to nothing: the tokens before the cut keep their
    values (but for a move to a larger scale), and the new ones follow.  Behind the new tokens the codes stay."""
    _need_gpu()
    s = Store(2, 2, ps, 4, 4, seed=40 + ps)
    for to, count, size in (([0] * 4, [50, 33, 64, 16], 1.0), ([37, 32, 0, 15], [2, 1, 3, 1], 0.01),
                            ([5, 20, 2, 0], [9, 30, 0, 7], 30.0), ([13, 47, 1, 3], [1, 1, 1, 1], 5.0)):
        s.n = list(to)
        k, v = s.rows(sum(count), kind, size)
        s.write(k, v, count)
        s.check()


@gpu
def test_tokens_behind_the_new_ones_are_lost():
    """The first tokens of a full block written again: the codes behind them stay and stand for other values."""
    _need_gpu()
    s = Store(1, 1, 16, 1, 1, seed=3)
    k, v = s.rows(16, "f32")
    s.write(k, v, [16])
    codes, scale = s.pool.clone(), s.sc.clone()
    s.n = [0]
    k, v = s.rows(4, "f32", 100.0)
    s.write(k, v, [4])
    s.check()
    at = int(s.table[0, 0])
    assert torch.equal(s.pool[0, at, 0, :, 4:], codes[0, at, 0, :, 4:])
    assert (s.sc[0, at] > scale[0, at]).all()
    out = [torch.empty((16, 1, 1, D), device="cuda") for _ in range(2)]
    md.md_read_cache8(out[0], out[1], s.pool, s.sc, s.bt, [0], [16])
    want = decode(codes[0, at, 0, 0, 4:].cpu().numpy()) * float(s.sc[0, at, 0, 0, 0])
    assert np.array_equal(out[0][4:, 0, 0].cpu().numpy(), want.astype(np.float32))
