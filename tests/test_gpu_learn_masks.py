"""The example that learns mask logits through the attention within packed sequences and the losses behind the logits: its list, its loss and its
gradients against the same chain in 64 bits."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F64 = torch.float64
PATTERNS = ((0, 1), (0, 2), (0, 3), (1, 2), (1, 3), (2, 3))        # the six candidates


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2509_23410_b200 import build
    build.build()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "learn_masks.py")
    spec = importlib.util.spec_from_file_location("learn_masks", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def masked(w, p_tile, p24, tau, kappa):
    """The soft mask without noise, times the weight."""
    n, k = w.shape
    s = torch.zeros(6, 4, dtype=F64, device="cuda")
    for c, at in enumerate(PATTERNS):
        s[c, list(at)] = 1.0
    tile = torch.sigmoid(kappa * p_tile / tau).repeat_interleave(128, 0).repeat_interleave(128, 1)
    group = (torch.softmax(kappa * p24 / tau, 0).T @ s).reshape(n, k)
    return (tile + (1 - tile) * group) * w.double()


def logits(block, x, bounds, positions, weights):
    Hq, Hkv, D = block.Hq, block.Hkv, block.D
    x = x.double()
    q, k, v = (x @ weights[0].T).unflatten(1, (-1, D)).split((Hq, Hkv, Hkv), 1)
    t = block.rope.table.double()[positions.long()]
    c, s = t[:, None, : D // 2], t[:, None, D // 2 :]

    def turned(h, w):
        h = h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6) * w.double()
        a, b = h[..., : D // 2], h[..., D // 2 :]
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    q, k = turned(q, block.wq), turned(k, block.wk).repeat_interleave(Hq // Hkv, 1)
    v, out = v.repeat_interleave(Hq // Hkv, 1), []
    for lo, hi in zip(bounds, bounds[1:]):
        e = torch.einsum("ihd,jhd->hij", q[lo:hi], k[lo:hi]) * D ** -0.5
        e = e.masked_fill(torch.ones(hi - lo, hi - lo, dtype=torch.bool, device="cuda").triu(1), -float("inf"))
        out.append(torch.einsum("hij,jhd->ihd", e.softmax(-1), v[lo:hi]))
    o = torch.cat((*out, torch.zeros(x.shape[0] - bounds[-1], Hq, D, dtype=F64, device="cuda")))
    return (x + o.flatten(1) @ weights[1].T) @ block.out.double().T[:, : block.V]


@pytest.mark.parametrize("hidden,Hq,Hkv,D,V,M,lens,k,rest", [(256, 4, 2, 64, 1000, 300, (130, 1, 97, 60), 20, True), (256, 2, 2, 128, 773, 129, (129,), 1, False),
                                                             (512, 8, 1, 128, 4097, 411, (1, 2, 3, 4, 400), 100, True)])
def test_gradients_of_the_mask_logits(example, hidden, Hq, Hkv, D, V, M, lens, k, rest):
    """A gradient passes at most fourteen roundings to bf16 on its way there and back (weight, projection, norm and rotation, probabilities, result,
    o projection, sum, logits; their gradient, both losses' sum, and the gradients of the sum's operands, of result, scores, projection and weight): each
    moves it by up to 2^-8 of its norm, so that 6e-2 covers them; the soft mask adds 1e-3 in a mask's value.  The loss: logits are of the size of one, so
    that 2^-8 of them, four times rounded on the way, is 2e-2 for a single row and less for the mean."""
    from paper_2509_23410_b200 import binding as B
    tau, kappa, temperature, share = 2.0, 1.5, 1.5, 0.5
    block = example.Block(hidden, Hq, Hkv, D, V, M)
    x, starts, tokens = example.batch(M, lens, hidden, V)
    loss, got, (ids, logp) = example.step(block, x, starts, tokens, k, temperature, share, rest, tau, kappa, flags=B.MASK_NO_NOISE)

    counts, positions = tokens >= 0, example.positions_of(starts, M)
    bounds = starts.tolist()
    with torch.no_grad():                                          # the list: the largest of the teacher's own logits, in order
        teacher = block.logits(x, starts, positions, block.W)
        top = teacher.double().topk(k, -1).values
        assert torch.equal(teacher.double().gather(1, ids.long().clamp(min=0))[counts], top[counts])
        assert bool((ids[~counts] == -1).all())
        want = torch.log_softmax(logits(block, x, bounds, positions, [w.double() for w in block.W]) / temperature, -1)
        want = want.gather(1, ids.long().clamp(min=0))
        assert float((logp.double() - want)[counts].abs().max()) < 0.1         # of 8 of the logits' standard deviation: 2^-8 of it, four times rounded

    leaves = [p.detach().double().requires_grad_() for pair in block.masks for p in pair]
    weights = [masked(w, leaves[2 * i], leaves[2 * i + 1], tau, kappa) for i, w in enumerate(block.W)]
    z = logits(block, x, bounds, positions, weights)
    lp = torch.log_softmax(z / temperature, -1)
    q = logp.double().exp()
    picked = lp.gather(1, ids.long().clamp(min=0))
    if rest:
        p_rest = 1 - picked.exp().sum(-1)
        per_row = -(q * picked).sum(-1) - (1 - q.sum(-1)).clamp(min=0) * torch.log(p_rest)
    else:
        per_row = -(q / q.sum(-1, keepdim=True) * picked).sum(-1)
    own = torch.log_softmax(z, -1).gather(1, tokens.clamp(min=0)[:, None])[:, 0]
    want = (share * per_row - (1 - share) * own)[counts].sum() / counts.sum()
    assert abs(float(loss) - float(want.detach())) < 2e-2
    for a, b in zip(got, torch.autograd.grad(want, leaves)):
        assert a.shape == b.shape and float((a.double() - b).norm() / b.norm()) < 6e-2


def test_step_again_and_on_another_stream(example):
    """Equal steps give equal bits, on any stream, and other noise another gradient."""
    block = example.Block(256, 4, 2, 64, 1000, 300)
    args = example.batch(300, (130, 1, 97, 60), 256, 1000)
    loss, grads, _ = example.step(block, *args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loss2, grads2, _ = example.step(block, *args)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(loss, loss2) and all(torch.equal(a, b) for a, b in zip(grads, grads2))
    _, grads3, _ = example.step(block, *args, seed=5)
    assert not any(torch.equal(a, b) for a, b in zip(grads, grads3))


def test_main(example, capsys):
    example.main()
    assert "ms a step" in capsys.readouterr().out
