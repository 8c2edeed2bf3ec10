"""The example on caches in eight bits runs at a small size."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_eight_bit_decode_example(capsys):
    if not torch.cuda.is_available():  # pragma: no cover
        pytest.skip("needs a CUDA GPU")
    spec = importlib.util.spec_from_file_location("eight_bit_decode", os.path.join(ROOT, "examples", "eight_bit_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    off = m.main(["--agents", "3", "--tokens", "2500", "--steps", "4", "--layers", "3", "--window", "300"])
    # elements are off by at most 2^-4 of themselves, or 2^-10 of a scale, which is 2^-7 of the block's largest at most
    assert off <= 2.0 ** -4 + 128 ** 0.5 * 2.0 ** -17 and "nan" not in capsys.readouterr().out
