"""The example that runs the attention-side operators between the packed linear layers, at small sizes."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2509_23410_b200 import build
    build.build()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")
    spec = importlib.util.spec_from_file_location("attention_layer", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("shape", [(512, 4, 4, 128, 3, 37, 5), (512, 8, 2, 64, 40, 130, 2), (1024, 8, 1, 128, 5, 300, 18)])
def test_prompt_and_steps(example, shape):
    """Rounding: queries, keys and probabilities to bf16 (2^-8 each at most, a third of that on average) and the result once more:
    1e-2 in the norm covers the four together."""
    hidden, Hq, Hkv, D, batch, prompt, steps = shape
    layer = example.Layer(hidden, Hq, Hkv, D, batch, max_prompt=prompt, max_own=32)
    assert example.serve(layer, prompt, steps) < 1e-2


def test_training(example):
    losses = example.train_step()
    assert losses[-1] < 0.2 * losses[0] and all(b < a for a, b in zip(losses, losses[1:]))
