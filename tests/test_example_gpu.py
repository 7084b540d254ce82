"""The example trains: the operators' gradients and the outer step together lower the
validation loss of the merged model."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_diloco_rounds():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("diloco_rounds", os.path.join(ROOT, "examples", "diloco_rounds.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.main(["--rounds", "3", "--workers", "2", "--inner-steps", "25", "--vocab", "256", "--dim", "96",
                           "--hidden", "250", "--blocks", "1"])
    # a uniform guess has log 256 = 5.5; the source's own entropy is about 0.9
    assert abs(losses[0] - math.log(256)) < 0.5
    assert losses[-1] < 0.5 * losses[0]
    assert all(math.isfinite(x) for x in losses)
