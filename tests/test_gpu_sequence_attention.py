"""Causal attention within packed sequences and its gradient against the definition in 64 bits, one sequence at a time.

Tolerances, b = 2^-8 (half a step of bf16).  A probability is rounded to bf16 for its product with V (the sum that divides takes it unrounded), the result
once: |O - o| <= b sum p |v| + b |o|.  Gradients: p and gs are rounded for their products, results once: b sum |gs| |k| + b |gq|, and so on.
What fp32 does (scores, exponents of size |lse|, sums of some thousand terms) is below 2^-15 of sum p |v|.  gp and delta are fp32 sums of D <= 128 products, off by
up to D 2^-24 = 2^-17 of sum |go| |v| and sum |go| |o| (not of their own values, which may cancel: in a row that sees one key their difference is 0
but for this): 2^-15 of p (|go| . |v| + |go| . |o|) covers both and p's own error."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
BF, F64 = torch.bfloat16, torch.float64
HALF, FINE = 2.0 ** -8, 2.0 ** -15


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2509_23410_b200 import build, binding as b
    build.build()
    return b


class Packed:
    """Sequences of the given lengths in a stacked projection whose other rows and columns are NaN."""

    def __init__(self, lens, Hq, Hkv, D, seed=0, lead=0, tail=0, scale=1.0, extra=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.Hq, self.Hkv, self.D, self.lead = lens, Hq, Hkv, D, lead
        n = sum(lens)
        self.M, width = lead + n + tail, (Hq + 2 * Hkv) * D
        self.bounds = [lead + sum(lens[:i]) for i in range(len(lens) + 1)]
        self.starts = torch.tensor(self.bounds, dtype=torch.int32, device="cuda")
        self.inside = torch.zeros(self.M, dtype=torch.bool, device="cuda")
        self.inside[lead : lead + n] = True

        def stack(w, s):
            x = torch.full((self.M, w + extra), math.nan, dtype=BF, device="cuda")
            x[self.inside, :w] = (s * torch.randn(n, w, generator=g, device="cuda")).to(BF)
            return x
        qkv = stack(width, scale)
        self.q, self.k, self.v = self.split(qkv)
        self.go = stack(Hq * D, 1.0)[:, : Hq * D].unflatten(1, (Hq, D))

    def split(self, x):
        Hq, Hkv, D = self.Hq, self.Hkv, self.D
        return (x[:, : Hq * D].unflatten(1, (Hq, D)), x[:, Hq * D : (Hq + Hkv) * D].unflatten(1, (Hkv, D)),
                x[:, (Hq + Hkv) * D : (Hq + 2 * Hkv) * D].unflatten(1, (Hkv, D)))

    def heads(self, x, a, b):
        x = x[a:b].to(F64).transpose(0, 1)
        return x.repeat_interleave(self.Hq // x.shape[0], 0)

    def each(self, scale):
        """(rows, p [Hq, n, n], lse [Hq, n], q, k, v by query head) of every sequence."""
        for a, b in zip(self.bounds, self.bounds[1:]):
            if a == b:
                continue
            q, k, v = (self.heads(x, a, b) for x in (self.q, self.k, self.v))
            s = (q @ k.transpose(1, 2)) * scale
            s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1), -math.inf)
            lse = s.logsumexp(-1)
            yield a, b, (s - lse[..., None]).exp(), lse, q, k, v


def close(got, want, tol, what):
    bad = ~((got.to(F64) - want).abs() <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), float((got.to(F64) - want).abs()[bad].max()), float(tol[bad].max()))


def check_forward(x, o, lse, scale):
    for a, b, p, want_lse, q, k, v in x.each(scale):
        want, size = (p @ v).transpose(0, 1), (p @ v.abs()).transpose(0, 1)
        close(o[a:b], want, HALF * (size + want.abs()) + FINE * size + 1e-30, "o")
        if lse is not None:
            close(lse[a:b], want_lse.t(), 2.0 ** -20 * (want_lse.t().abs() + 4), "lse")


def check_backward(x, o, lse, grads, scale):
    group = lambda y: y.view(x.Hkv, x.Hq // x.Hkv, *y.shape[1:]).sum(1).transpose(0, 1)  # noqa: E731
    for a, b, p, _, q, k, v in x.each(scale):
        go, oo = x.heads(x.go, a, b), x.heads(o, a, b)
        p = (((q @ k.transpose(1, 2)) * scale) - lse[a:b].to(F64).t()[..., None]).exp().tril()         # the call's inputs are its own lse and O
        gp, delta = go @ v.transpose(1, 2), (go * oo).sum(-1, keepdim=True)
        gs = p * (gp - delta) * scale
        fine = FINE * p * (go.abs() @ v.abs().transpose(1, 2) + (go * oo).abs().sum(-1, keepdim=True)) * scale
        want, size = gs @ k, gs.abs() @ k.abs()
        close(grads[0][a:b], want.transpose(0, 1), (HALF * (size + want.abs()) + fine @ k.abs() + 1e-30).transpose(0, 1), "gq")
        want, size = group(gs.transpose(1, 2) @ q), group(gs.abs().transpose(1, 2) @ q.abs())
        close(grads[1][a:b], want, HALF * (size + want.abs()) + group(fine.transpose(1, 2) @ q.abs()) + 1e-30, "gk")
        want, size = group(p.transpose(1, 2) @ go), group(p.transpose(1, 2) @ go.abs())
        close(grads[2][a:b], want, HALF * (size + want.abs()) + FINE * size + 1e-30, "gv")


def run(B, x, scale=None, backward=True):
    real = x.D ** -0.5 if scale is None else scale
    o, lse = torch.full((x.M, x.Hq, x.D), 5.0, dtype=BF, device="cuda"), torch.full((x.M, x.Hq), 5.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.patch_sequence_attention(x.q, x.k, x.v, x.starts, scale=scale, O=o, lse=lse, status=status)
    check_forward(x, o, lse, real)
    assert bool((o[~x.inside] == 5.0).all()) and bool((lse[~x.inside] == 5.0).all()), "rows outside the sequences"
    assert int(status) == 0
    if not backward:
        return o, lse
    o[~x.inside], lse[~x.inside] = math.nan, math.nan
    grads = x.split(torch.full((x.M, (x.Hq + 2 * x.Hkv) * x.D), 5.0, dtype=BF, device="cuda"))
    B.patch_sequence_attention_backward(x.go, x.q, x.k, x.v, o, lse, x.starts, scale=scale, gQ=grads[0], gK=grads[1], gV=grads[2], status=status)
    check_backward(x, o, lse, grads, real)
    assert all(bool((y[~x.inside] == 5.0).all()) for y in grads), "rows outside the sequences"
    assert int(status) == 0
    return o, lse, grads


LENGTHS = [[1], [2], [63], [64], [65], [127], [128], [129], [255, 257], [1, 0, 1, 200, 0, 0, 33], [300, 5, 129, 128, 64, 1, 77], [0], [0, 0, 3], [511, 130], [1] * 40, [1025]]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda v: "-".join(map(str, v))[:24])
def test_lengths(B, D, lens):
    run(B, Packed(lens, 4, 2, D, seed=len(lens)))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (8, 1), (6, 3), (5, 5), (16, 2), (7, 1)])
def test_heads(B, D, Hq, Hkv):
    run(B, Packed([200, 70, 131], Hq, Hkv, D, seed=Hq))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lead,tail,extra", [(1, 0, 0), (0, 1, 8), (77, 300, 64), (128, 128, 0)])
def test_rows_around_the_sequences(B, D, lead, tail, extra):
    run(B, Packed([5, 130, 0, 64], 4, 2, D, seed=3, lead=lead, tail=tail, extra=extra))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [0.01, 0.5])
def test_scales_and_sharp_rows(B, D, scale):
    run(B, Packed([300, 129], 4, 2, D, seed=4, scale=2.0), scale=scale)


@pytest.mark.parametrize("D", [64, 128])
def test_long(B, D):
    run(B, Packed([2500, 700], 4, 1, D, seed=6, scale=1.3))


@pytest.mark.parametrize("n", [127, 128, 129, 200, 1000])
def test_many_sequences(B, n):
    """Items are taken by size up to a number of sequences, one sequence behind the other beyond it."""
    lens = [(0, 1, 7, 128, 129, 260, 33)[(5 * i + i // 7) % 7] for i in range(n)]
    run(B, Packed(lens, 2, 1, 64, seed=n, lead=3, tail=5))


@pytest.mark.parametrize("D,Hq,Hkv,n", [(64, 128, 128, 128), (128, 96, 48, 60), (64, 140, 70, 400)])
def test_groups_of_heads(B, D, Hq, Hkv, n):
    """More heads than are taken together; the last group may be smaller."""
    run(B, Packed([(9 * i) % 53 + 200 * (i % 15 == 2) for i in range(n)], Hq, Hkv, D, seed=n))


def test_nan_stays_in_its_sequence(B):
    x = Packed([130, 70, 200], 4, 2, 128, seed=5)
    x.q[140], x.k[150], x.v[160], x.go[170] = math.nan, math.inf, math.nan, math.nan
    o, lse = torch.empty(x.M, 4, 128, dtype=BF, device="cuda"), torch.empty(x.M, 4, device="cuda")
    B.patch_sequence_attention(x.q, x.k, x.v, x.starts, O=o, lse=lse)
    grads = B.patch_sequence_attention_backward(x.go, x.q, x.k, x.v, o, lse, x.starts)
    other = torch.ones(x.M, dtype=torch.bool, device="cuda")
    other[130:200] = False
    assert all(not bool(y[other].isnan().any()) for y in (o, lse, *grads))


@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_any_size(B, D):
    """A row's largest score wins outright, at scores up to 2^100; the result is its value."""
    x = Packed([400], 2, 1, D, seed=8)
    x.q.copy_(2.0 ** 50 * torch.sign(torch.randn(400, 2, D, device="cuda")))
    x.k.copy_(2.0 ** 40 * torch.randn(400, 1, D, device="cuda").to(BF))
    o = B.patch_sequence_attention(x.q, x.k, x.v, x.starts)
    s = torch.einsum("ihd,jd->hij", x.q.to(F64), x.k[:, 0].to(F64)).masked_fill(torch.ones(400, 400, dtype=torch.bool, device="cuda").triu(1), -math.inf)
    top = s.topk(2, -1)
    gap = (top.values[..., 0] - top.values[..., 1]).t() > 2.0 ** 70                 # fp32 sums of this size are off by less
    want = x.v[:, 0][top.indices[..., 0].t()]
    assert bool(gap.float().mean() > 0.9) and torch.equal(o[gap], want[gap])


def test_ascending_scores(B):
    """Maxima that rise from key to key, from tile to tile."""
    x = Packed([900], 2, 2, 64, seed=9)
    ramp = torch.linspace(0, 24, 900, device="cuda")[:, None, None]
    x.k.copy_((x.k.float() * 0.1 + ramp).to(BF))
    x.q.copy_((x.q.float() * 0.1 + 1.0).to(BF))
    run(B, x)
    x.k.copy_(x.k.flip(0))
    run(B, x)


def test_gradient_against_differences(B):
    """d/dt of sum(c o) along random directions: bf16 inputs on a grid so that both sides of the difference are exact."""
    M, H, D, h = 40, 2, 64, 2.0 ** -4
    g = torch.Generator(device="cuda").manual_seed(2)
    draw = lambda: (torch.randint(-16, 17, (M, H, D), generator=g, device="cuda") / 16.0)  # noqa: E731
    q, k, v, c, dq, dk, dv = (draw() for _ in range(7))
    starts = torch.tensor([0, 25, 40], dtype=torch.int32, device="cuda")

    def f(t):
        o = B.patch_sequence_attention((q + t * dq).to(BF), (k + t * dk).to(BF), (v + t * dv).to(BF), starts)
        return (o.double() * c).sum()
    lse = torch.empty(M, H, device="cuda")
    o = B.patch_sequence_attention(q.to(BF), k.to(BF), v.to(BF), starts, lse=lse)
    gq, gk, gv = B.patch_sequence_attention_backward(c.to(BF), q.to(BF), k.to(BF), v.to(BF), o, lse, starts)
    got, want = float((gq.double() * dq + gk.double() * dk + gv.double() * dv).sum()), float((f(h) - f(-h)) / (2 * h))
    # roundings of 2 M H D results, random in sign: b |o| |c| sqrt(2 M H D) / (2 h); the gradients' own; the third derivative
    assert abs(got - want) < 4 * HALF * 0.5 * 0.6 * math.sqrt(2 * M * H * D) / (2 * h) + 0.02 * abs(want)


def test_starts_out_of_order_or_range_are_reported(B):
    x = Packed([100, 60], 2, 1, 64, seed=1)
    for bad in ([0, 100, 400], [-5, 100, 160], [0, 100, 50], [100, 0, 160], [2 ** 31 - 1, -2 ** 31, 7]):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        starts = torch.tensor(bad, dtype=torch.int32, device="cuda")
        o, lse = torch.zeros(160, 2, 64, dtype=BF, device="cuda"), torch.zeros(160, 2, device="cuda")
        B.patch_sequence_attention(x.q, x.k, x.v, starts, O=o, lse=lse, status=status)
        assert int(status) == B.ERR_SIZE, bad
        status.zero_()
        B.patch_sequence_attention_backward(x.go, x.q, x.k, x.v, o, lse, starts, status=status)
        assert int(status) == B.ERR_SIZE, bad
    run(B, x)


def test_equal_calls_give_equal_bits(B):
    x = Packed([300, 513, 64], 8, 2, 128, seed=2)
    first = run(B, x)
    for _ in range(3):
        again = run(B, x)
        assert torch.equal(first[0][x.inside], again[0][x.inside]) and all(torch.equal(a, b) for a, b in zip(first[2], again[2]))


def test_captured_calls_follow_their_starts(B):
    x = Packed([300, 84], 4, 2, 128, seed=2)
    o, lse = torch.empty(x.M, 4, 128, dtype=BF, device="cuda"), torch.empty(x.M, 4, device="cuda")
    grads = [torch.empty(x.M, h, 128, dtype=BF, device="cuda") for h in (4, 2, 2)]
    ws = torch.empty(B.patch_sequence_attention_backward_workspace_size(x.M, 2, 4, 2, 128), dtype=torch.uint8, device="cuda")

    def step():
        B.patch_sequence_attention(x.q, x.k, x.v, x.starts, O=o, lse=lse)
        B.patch_sequence_attention_backward(x.go, x.q, x.k, x.v, o, lse, x.starts, gQ=grads[0], gK=grads[1], gV=grads[2], workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([300, 84], [1, 383], [384, 0], [200, 184]):
        x.lens, x.bounds = lens, [0, lens[0], 384]
        x.starts.copy_(torch.tensor(x.bounds, dtype=torch.int32))
        graph.replay()
        check_forward(x, o, lse, 128 ** -0.5)
        check_backward(x, o, lse, grads, 128 ** -0.5)


def test_two_streams_at_once(B):
    xs = [Packed([700, 300], 8, 2, 128, seed=s) for s in (1, 2)]
    want = [run(B, x) for x in xs]
    side = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for x, s in zip(xs, side):
            lse = torch.empty(x.M, 8, device="cuda")
            o = B.patch_sequence_attention(x.q, x.k, x.v, x.starts, lse=lse, stream=s)
            got.append((o, B.patch_sequence_attention_backward(x.go, x.q, x.k, x.v, o, lse, x.starts, stream=s), lse))
    torch.cuda.synchronize()
    for i, (o, grads, _) in enumerate(got):
        assert torch.equal(o, want[i % 2][0]) and all(torch.equal(a, b) for a, b in zip(grads, want[i % 2][2]))


def test_offsets_beyond_32_bits(B):
    """Rows whose elements are numbered beyond 2^32."""
    n, ld = 300, 1 << 24
    free, _ = torch.cuda.mem_get_info()
    if free < n * ld * 2 * 2:
        pytest.skip("needs 20 GB")
    x = Packed([170, 130], 2, 1, 64, seed=7)
    wide = torch.empty(n, ld, dtype=BF, device="cuda")[:, : 4 * 64]
    wide.copy_(torch.cat([y.flatten(1) for y in (x.q, x.k, x.v)], 1))
    x.q, x.k, x.v = x.split(wide)
    run(B, x)


def test_nothing_to_do(B):
    q = torch.zeros(0, 2, 64, dtype=BF, device="cuda")
    starts = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert B.patch_sequence_attention(q, q, q, starts).shape == (0, 2, 64)
    x = Packed([0, 0], 2, 2, 64, tail=70)
    run(B, x)
    o = torch.full((70, 2, 64), 3.0, dtype=BF, device="cuda")
    B.patch_sequence_attention(x.q, x.k, x.v, starts[:1], O=o)
    assert bool((o == 3.0).all())


def test_refusals_of_the_binding(B):
    x = Packed([40], 2, 1, 64)
    for q, k, v, starts in ((x.q.float(), x.k, x.v, x.starts), (x.q, x.k[:39], x.v, x.starts), (x.q, x.k, x.q, x.starts), (x.q, x.k, x.v, x.starts.long()),
                            (x.q, x.k, x.v, x.starts[:0]), (x.q.cpu(), x.k, x.v, x.starts), (x.q, x.k, x.v, x.starts.cpu())):
        with pytest.raises(AssertionError):
            B.patch_sequence_attention(q, k, v, starts)
    with pytest.raises(B.PatchError):
        B.patch_sequence_attention(x.q, x.k, x.v, x.starts, scale=-1.0)
    with pytest.raises(B.PatchError):
        B.patch_sequence_attention(*(torch.zeros(40, 1, 32, dtype=BF, device="cuda") for _ in range(3)), x.starts)
