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


@pytest.mark.parametrize("norms", [(False, False), (True, False), (False, True), (True, True)])
def test_autograd_function(example, norms):
    """With either weight left out, and differentiated once only.  Results and gradients are rounded to bf16: 2^-8 each."""
    M, Hq, Hkv, D = 20, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    tab = example.rope_table(M, D)
    rope, pos = example.B.patch_rope(tab), torch.arange(M, dtype=torch.int32, device="cuda")
    x = [rand(M, Hq, D).requires_grad_(), rand(M, Hkv, D).requires_grad_()]
    w = [(1 + 0.1 * rand(D)).requires_grad_() if n else None for n in norms]
    gy = [rand(M, Hq, D), rand(M, Hkv, D)]
    leaves = x + [t for t in w if t is not None]
    got = torch.autograd.grad(sum((y * t).sum() for y, t in zip(example.QKNormRope.apply(*x, *w, rope, pos, 1e-6), gy)), leaves)
    leaves64 = [t.detach().double().requires_grad_() for t in leaves]
    loss, weights, c, s = 0.0, iter(leaves64[2:]), tab[:, None, : D // 2].double(), tab[:, None, D // 2 :].double()
    for y, norm, t in zip(leaves64[:2], norms, gy):
        if norm:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6) * next(weights)
        a, b = y[..., : D // 2], y[..., D // 2 :]
        loss = loss + (torch.cat((a * c - b * s, b * c + a * s), -1) * t.double()).sum()
    for a, b in zip(got, torch.autograd.grad(loss, leaves64)):
        assert float((a.double() - b).norm() / b.norm()) < 1e-2
    y, _ = example.QKNormRope.apply(*x, *w, rope, pos, 1e-6)
    (gx,) = torch.autograd.grad(y.float().square().sum(), x[:1], create_graph=True)
    with pytest.raises(RuntimeError):
        gx.float().square().sum().backward()
