"""Scores at their ends: rows whose maximum moves from part to part of a tile, and finite scores of any size.

The block kernel raises a row's maximum only where a half of a tile (64 keys) sums to more than 256, so its inputs here are made to: keys
along one direction that all queries have in common, in steps of 64 keys from one half to the next.  Tolerances of ``Batch.check`` (derived
there) hold: they grow with the scores' sizes.  Where scores are huge the softmax is a choice: every product is exact, two different
scores are more than 2^12 powers of two apart, so the result is the mean of the values of the largest score's keys."""
import random

import pytest

torch = pytest.importorskip("torch")
from test_gpu_attention import BF, B, Batch  # noqa: E402,F401  (B is a fixture)

pytestmark = pytest.mark.gpu

# lens, T, Hq, Hkv, D, P, page, extra pages in the table
BLOCK = [
    ([5] * 33, 1, 8, 2, 128, 16000, 16, 0),                # the prefix: 132 rows in two blocks
    ([3] * 20, 1, 4, 4, 64, 33003, 64, 0),                 # a block of 20 rows
    ([700, 64], 600, 1, 1, 128, 300, 16, 10000),           # prompts, behind a prefix and without
    ([640], 520, 2, 1, 64, 0, 32, 5000),
    ([513, 1000], 40, 4, 2, 128, 0, 128, 1250),
]


def refill(x):
    """The batch's keys into its pages again."""
    used = x.prefix_pages.tolist()
    x._put(used, x.kp, x.vp)
    table = x.table.tolist()
    for b, n in enumerate(x.lens):
        x._put(table[b][: -(-n // x.page)], x.ks[b], x.vs[b])


def stairs(x, seed, step=4.5):
    """Keys along a direction that the queries share: in every half of a tile of the prefix's and of each sequence's keys (counted from
    their first), or in none, the scores go up by `step` powers of two."""
    rng = random.Random(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    D = x.D
    u = torch.where(torch.rand(D, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    x.q = (u + 0.05 * torch.randn(x.q.shape, generator=g, device="cuda")).to(BF)
    ups = []

    def keys(n):
        half, levels, level = (n + 63) // 64, [], 0.0
        for i in range(half):
            ups.append(i > 0 and rng.random() < 0.6)
            level += step if ups[-1] else 0.0
            levels.append(level)
        at = torch.tensor(levels or [0.0], device="cuda")[torch.arange(n, device="cuda") // 64]
        return (at[:, None, None] / (D ** 0.5 * 1.4427) * u + 0.02 * torch.randn(n, x.Hkv, D, generator=g, device="cuda")).to(BF)
    x.kp = keys(x.P)
    x.ks = [keys(n) for n in x.lens]
    refill(x)
    return ups


@pytest.mark.parametrize("case", range(len(BLOCK)))
@pytest.mark.parametrize("seed", range(3))
def test_block_kernel_raises_the_maximum(B, case, seed):
    lens, T, Hq, Hkv, D, P, page, extra = BLOCK[case]
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case, extra=extra)
    stairs(x, 10 * case + seed)
    o, l = x.run(B)
    x.check(o, l)
    o2, _ = x.run(B, lse=False)
    assert torch.equal(o, o2), "equal calls give equal bits"


@pytest.mark.parametrize("case", range(len(BLOCK)))
@pytest.mark.parametrize("q_scale", [8.0, 40.0])
def test_block_kernel_with_peaked_scores(B, case, q_scale):
    """Scores of random keys far apart, and keys that grow along the sequence."""
    lens, T, Hq, Hkv, D, P, page, extra = BLOCK[case]
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case, q_scale=q_scale, extra=extra)
    grow = lambda k: (k.float() * (0.05 + 2.0 * torch.arange(k.shape[0], device="cuda")[:, None, None] / max(1, k.shape[0]))).to(BF)  # noqa: E731
    x.kp, x.ks = grow(x.kp), [grow(k) for k in x.ks]
    refill(x)
    o, l = x.run(B)
    x.check(o, l)


def choose(x, power, seed):
    """Scores q.k = 2^power k0 with whole k0 from -6 to 6: exact in fp32 (one product), ties included."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    e = lambda n: torch.randint(-6, 7, (n, x.Hkv), generator=g, device="cuda").float()  # noqa: E731

    def keys(n):
        k = torch.zeros(n, x.Hkv, x.D, device="cuda")
        k[..., 0] = e(n)
        return k.to(BF)
    x.kp, x.ks = keys(x.P), [keys(n) for n in x.lens]
    refill(x)
    q = torch.zeros(x.q.shape, device="cuda")
    q[..., 0] = torch.where(torch.rand(x.q.shape[:2], generator=g, device="cuda") < 0.5, -1.0, 1.0) * 2.0 ** power
    x.q = q.to(BF)


def check_chosen(x, o, l):
    G, T = x.Hq // x.Hkv, x.T
    for b in range(len(x.lens)):
        k = torch.cat((x.kp, x.ks[b]))[..., 0].double().transpose(0, 1)                  # [Hkv, n]
        v = torch.cat((x.vp, x.vs[b])).double().transpose(0, 1)
        for t in range(T):
            n, row = x.P + max(0, x.lens[b] - (T - 1 - t)), b * T + t
            if n == 0:
                continue
            s = x.q[row, :, 0].double().view(x.Hkv, G, 1) * k[:, None, :n]
            top = s.amax(-1, keepdim=True)
            p = (s == top).double()
            want = torch.einsum("hgn,hnd->hgd", p, v[:, :n]) / p.sum(-1, keepdim=True)
            size = torch.einsum("hgn,hnd->hgd", p, v[:, :n].abs()) / p.sum(-1, keepdim=True)
            # probabilities of 1 or of one power of two: only the result is rounded, and sums in fp32
            tol = want.abs() * 2.0 ** -8 * 1.01 + size * 2.0 ** -15 + 1e-30
            err = (o[row].double().view(x.Hkv, G, x.D) - want).abs()
            assert bool((err <= tol).all()), (b, t, float((err / tol).nan_to_num(1e9).max()))
            # a rounding each: the root of D, its reciprocal, log2(e), its product with the scale, that with the score, the sum with
            # log2 of the number of ties, ln 2 and its product with the sum
            want = (top.squeeze(-1) * x.D ** -0.5 + p.sum(-1).log()).view(-1)
            assert bool(((l[row].double() - want).abs() <= want.abs() * 8 * 2.0 ** -24 + 1e-5).all())


POWERS = [16, 24, 28, 29, 30, 31, 32, 33, 34, 38, 60, 100, 120]


SHAPES = BLOCK + [
    ([100, 333], 1, 8, 2, 128, 200, 16, 0),                # the single launch
    ([300, 0, 64], 2, 8, 1, 64, 64, 32, 0),
    ([90], 64, 3, 3, 128, 5, 32, 0),
    ([100, 333, 5], 1, 8, 2, 128, 2000, 16, 10000),        # decode kernel
    ([700, 64, 1], 4, 8, 2, 64, 0, 32, 5000),
    ([40] * 20, 1, 4, 4, 128, 1000, 16, 10000),
]


@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_scores_of_any_size(B, case):
    """Finite scores, however large (rows of a padded batch may hold anything finite): no row vanishes, none becomes NaN."""
    lens, T, Hq, Hkv, D, P, page, extra = SHAPES[case]
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case, extra=extra)
    for power in POWERS:
        choose(x, power, power)
        o, l = x.run(B)
        check_chosen(x, o, l)


@pytest.mark.parametrize("case", range(len(BLOCK), len(SHAPES)))
def test_moving_maximum(B, case):
    lens, T, Hq, Hkv, D, P, page, extra = SHAPES[case]
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case, extra=extra)
    stairs(x, case)
    o, l = x.run(B)
    x.check(o, l)


@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_a_query_that_is_not_a_number_shows(B, case):
    """NaN in a query makes its result and its lse NaN (not the 0 and -inf of a row that sees nothing) and leaves all others alone."""
    lens, T, Hq, Hkv, D, P, page, extra = SHAPES[case]
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case, extra=extra)
    want, want_l = x.run(B)
    rows = {(b * T + t, (b + t) % Hq) for b in range(len(lens)) for t in (0, T - 1)}
    mask = torch.zeros(x.q.shape[:2], dtype=torch.bool, device="cuda")
    for row, h in rows:
        x.q[row, h, (7 * row) % D] = float("nan")
        b, t = divmod(row, T)
        mask[row, h] = P + max(0, lens[b] - (T - 1 - t)) > 0          # a row without keys stays 0
    o, l = x.run(B)
    assert bool(mask.any()) and bool(o[mask].isnan().all()) and bool(l[mask].isnan().all())
    assert torch.equal(o[~mask], want[~mask]) and torch.equal(l[~mask], want_l[~mask])
