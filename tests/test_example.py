"""The example program runs at a small size."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_sparse_decode_example(capsys):
    if not torch.cuda.is_available():  # pragma: no cover
        pytest.skip("needs a CUDA GPU")
    spec = importlib.util.spec_from_file_location("sparse_decode", os.path.join(ROOT, "examples", "sparse_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.main(["--agents", "3", "--tokens", "2500", "--steps", "4", "--top", "8", "--layers", "2"])
    assert set(r) == {0, 8} and "nan" not in capsys.readouterr().out
