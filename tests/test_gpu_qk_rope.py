"""Norms and rotation of queries and keys, their gradient, and the paged append on the GPU, against the formulas in
64 bits.

Tolerances.  A result is one bf16 rounding (at most 2^-8 of its size) of an fp32 evaluation; the fp32 part has a sum of at most 256
squares and about ten roundings, each 2^-24 of the terms' sizes, so 2^-18 of the terms' sizes covers it.  A weight's
gradient is an fp32 sum: with at most 4096 terms in a thread's chain or across blocks, 4096 * 2^-24 of the sum of sizes bounds it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2509_23410_b200 import build, binding
    build.build()
    binding.lib()
    return binding


def table(n, R, seed=0):
    ang = torch.arange(n, dtype=torch.float64)[:, None] * (10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / max(R, 1)))[None]
    return torch.cat((ang.cos(), ang.sin()), 1).float().cuda()


def turn64(x, tab, pos, R, inter, back=False):
    """Rotation as it is written down: pair by pair, in 64 bits."""
    y = x.clone()
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + R // 2)
        c, s = tab[pos, i].double()[:, None], tab[pos, R // 2 + i].double()[:, None] * (-1 if back else 1)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def forward64(x, w, tab, pos, R, inter, eps):
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    return turn64(x, tab, pos, R, inter)


def sizes64(x, w, R, inter, eps):
    """Sizes of the terms of every result element."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    x = x.abs()
    return x + x.amax(-1, keepdim=True)


def check(got, ref, size, what):
    err = (got.double() - ref).abs()
    tol = ref.abs() * 2.0 ** -8 * 1.01 + size * 2.0 ** -18 + 1e-37
    assert bool((err <= tol).all()), (what, float((err / tol).max()))


def make(M, H, D, seed, pitch=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.randn(M, H * D + pitch, generator=g, device="cuda") * scale
    return buf.to(BF)[:, : H * D].unflatten(1, (H, D))


def weight(D, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(BF)


CASES = [  # M, Hq, Hkv, D, R, interleaved, norm q, norm k, pitch
    (1, 32, 32, 128, 128, False, True, True, 0),
    (1, 1, 1, 8, 0, False, True, True, 8),
    (3, 5, 1, 16, 16, False, True, True, 8),
    (2, 3, 2, 24, 16, False, True, False, 24),
    (7, 4, 4, 64, 64, False, False, False, 64),
    (7, 4, 2, 64, 32, True, True, True, 64),
    (33, 9, 3, 80, 80, False, True, True, 16),
    (33, 9, 3, 96, 24, True, False, True, 16),
    (129, 40, 40, 128, 64, False, True, True, 40 * 128),
    (64, 32, 8, 128, 128, True, True, True, 2048),
    (17, 6, 1, 256, 256, False, True, True, 0),
    (17, 6, 0, 192, 128, True, True, False, 0),
    (11, 0, 7, 256, 64, False, False, True, 0),
    (700, 32, 32, 128, 128, False, True, True, 4096),      # several heads per group of lanes
    (3001, 16, 2, 64, 64, False, True, True, 0),
]


@pytest.mark.parametrize("case", CASES)
def test_forward_and_backward(B, case):
    M, Hq, Hkv, D, R, inter, nq, nk, pitch = case
    q = make(M, Hq, D, 1, pitch) if Hq else None
    k = make(M, Hkv, D, 2, pitch, 3.0) if Hkv else None
    wq, wk = weight(D, 3) if nq else None, weight(D, 4) if nk else None
    tab = table(500, R) if R else None
    rope = B.patch_rope(tab, interleaved=inter) if R else None
    pos = torch.randint(0, 500, (M,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(5))
    p64 = pos.long()
    tb = tab if R else torch.zeros(500, 0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    qo, ko = B.patch_qk_norm_rope(q, k, rope, pos if R else None, wq=wq, wk=wk, eps=1e-5, status=status)
    for x, y, w in ((q, qo, wq), (k, ko, wk)):
        if x is not None:
            check(y, forward64(x, w, tb, p64, R, inter, 1e-5), sizes64(x, w, R, inter, 1e-5), "forward")
    gqo = make(M, Hq, D, 6, pitch) if Hq else None
    gko = make(M, Hkv, D, 7, pitch) if Hkv else None
    args = (gqo, gko, rope, pos if R else None)
    gq, gk, gwq, gwk = B.patch_qk_norm_rope_backward(*args, Q=q, K=k, wq=wq, wk=wk, eps=1e-5, status=status)
    for x, gy, gx, w, gw in ((q, gqo, gq, wq, gwq), (k, gko, gk, wk, gwk)):
        if x is None:
            continue
        g = turn64(gy.double(), tb, p64, R, inter, back=True)
        if w is None:
            check(gx, g, 2 * gy.double().abs().amax(-1, keepdim=True), "rotation back")
            assert gw is None
            continue
        x = x.double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
        xh, gn = x * r, g * w.double()
        ref = r * (gn - xh * (gn * xh).mean(-1, keepdim=True))
        big = r * (w.double().abs() * 2 * gy.double().abs().amax(-1, keepdim=True) + xh.abs() * (gn * xh).abs().mean(-1, keepdim=True))
        check(gx, ref, big, "gradient")
        ref, total = (g * xh).sum((0, 1)), (2 * gy.double().abs().amax(-1, keepdim=True) * xh.abs()).sum((0, 1))
        assert bool(((gw.double() - ref).abs() <= total * 2.0 ** -12).all())
        # what it really does is far nearer: chains of a few hundred terms whose roundings cancel
        assert float((gw.double() - ref).norm() / ref.norm()) < 1e-5
    again = B.patch_qk_norm_rope_backward(*args, Q=q, K=k, wq=wq, wk=wk, eps=1e-5, status=status)
    for a, b in zip((gq, gk, gwq, gwk), again):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b)), "equal calls give equal bits"
    assert int(status.item()) == 0


@pytest.mark.parametrize("inter", [False, True])
def test_gradient_against_differences(B, inter):
    """The gradient kernel against differences of the definition: L = sum(gy * y) along random directions."""
    M, H, D, R = 5, 3, 64, 32
    q, k = make(M, H, D, 11), make(M, 2, D, 12)
    wq, wk = weight(D, 13), weight(D, 14)
    tab = table(64, R)
    pos = torch.tensor([0, 1, 7, 63, 20], dtype=torch.int32, device="cuda")
    gqo, gko = make(M, H, D, 15), make(M, 2, D, 16)
    gq, gk, gwq, gwk = B.patch_qk_norm_rope_backward(gqo, gko, B.patch_rope(tab, inter), pos, Q=q, K=k, wq=wq, wk=wk, eps=1e-6)

    def loss(x, w, gy):
        return float((forward64(x, w, tab, pos.long(), R, inter, 1e-6) * gy.double()).sum())
    for x, w, gy, gx, gw in ((q, wq, gqo, gq, gwq), (k, wk, gko, gk, gwk)):
        for seed in range(3):
            dx = torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(20 + seed), device="cuda", dtype=torch.float64)
            dw = torch.randn(D, generator=torch.Generator(device="cuda").manual_seed(30 + seed), device="cuda", dtype=torch.float64)
            h = 1e-5
            want = (loss(x.double() + h * dx, w.double(), gy) - loss(x.double() - h * dx, w.double(), gy)) / (2 * h)
            got = float((gx.double() * dx).sum())
            # the results are rounded to bf16: 2^-8 of each term; the difference itself is good to h^2
            assert abs(got - want) <= float((gx.double() * dx).abs().sum()) * 2.0 ** -8 + 1e-6
            want = (loss(x.double(), w.double() + h * dw, gy) - loss(x.double(), w.double() - h * dw, gy)) / (2 * h)
            got = float((gw.double() * dw).sum())
            assert abs(got - want) <= float((gw.double() * dw).abs().sum()) * 2.0 ** -14 + 1e-6


def test_in_place_and_no_tokens(B):
    qkv = make(50, 12, 128, 1).reshape(50, 12 * 128).contiguous()
    q, k = qkv[:, : 8 * 128].unflatten(1, (8, 128)), qkv[:, 8 * 128 : 10 * 128].unflatten(1, (2, 128))
    before = qkv.clone()
    rope, pos, wq, wk = B.patch_rope(table(64, 128)), torch.arange(50, dtype=torch.int32, device="cuda"), weight(128, 1), weight(128, 2)
    qo, ko = B.patch_qk_norm_rope(q, k, rope, pos, wq=wq, wk=wk)
    B.patch_qk_norm_rope(q, k, rope, pos, wq=wq, wk=wk, Q_out=q, K_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, 10 * 128 :], before[:, 10 * 128 :])
    # the gradient in place of the results' gradient
    g = make(50, 8, 128, 3)
    gq, _, gwq, _ = B.patch_qk_norm_rope_backward(g, None, rope, pos, Q=qo, wq=wq)
    g2 = g.clone()
    _, _, gwq2, _ = B.patch_qk_norm_rope_backward(g2, None, rope, pos, Q=qo, wq=wq, gQ=g2)
    assert torch.equal(g2, gq) and torch.equal(gwq, gwq2)
    # no tokens: nothing is launched, the weights' gradients are zero
    e, epos = torch.empty(0, 8, 128, dtype=BF, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    B.patch_qk_norm_rope(e, None, rope, epos, wq=wq)
    gw = torch.full((128,), 7.0, device="cuda")
    B.patch_qk_norm_rope_backward(e, None, rope, epos, Q=e, wq=wq, gwq=gw)
    assert float(gw.abs().max()) == 0.0


def test_values_at_the_ends(B):
    """Rows of zeros (the norm divides by sqrt(eps)), of the largest values, and a row with NaN that stays in its row."""
    q = make(4, 2, 128, 1).contiguous()
    q[0] = 0
    q[1] = 1e18
    q[2, 1, 5] = float("nan")
    w, rope = weight(128, 2), B.patch_rope(table(8, 128))
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    y, _ = B.patch_qk_norm_rope(q, None, rope, pos, wq=w, eps=1e-6)
    assert float(y[0].abs().max()) == 0.0 and bool(torch.isfinite(y[1]).all())
    assert bool(torch.isnan(y[2, 1]).all()) and bool(torch.isfinite(y[2, 0]).all()) and bool(torch.isfinite(y[3]).all())
    # elements beyond the rotated part are untouched by it, infinities included
    q[3, 0, 100] = float("inf")
    y, _ = B.patch_qk_norm_rope(q, None, B.patch_rope(table(8, 64)), pos)
    assert torch.equal(y[3, 0, 64:], q[3, 0, 64:]) and bool(torch.isfinite(y[3, 0, :64]).all())


def test_positions_outside_the_table_are_reported(B):
    q = make(4, 2, 64, 1)
    rope = B.patch_rope(table(8, 64))
    for bad in (8, -1, 2 ** 31 - 1):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        pos = torch.tensor([1, 2, bad, 3], dtype=torch.int32, device="cuda")
        y, _ = B.patch_qk_norm_rope(q, None, rope, pos, status=status)
        assert int(status.item()) == B.ERR_SIZE
        ok, _ = B.patch_qk_norm_rope(q, None, rope, torch.where((pos < 0) | (pos > 7), 0, pos).int())
        assert torch.equal(y, ok)


@pytest.mark.parametrize("case", [(1, 32, 32, 128, 128, 16, True), (5, 8, 2, 64, 32, 64, False), (300, 40, 40, 128, 128, 16, False),
                                  (77, 6, 3, 96, 96, 32, True), (2100, 16, 2, 64, 64, 128, True), (9, 4, 1, 256, 0, 256, True)])
def test_append(B, case):
    M, Hq, Hkv, D, R, page, norm = case
    x = make(M, Hq + 2 * Hkv, D, 1)
    q, k, v = x[:, :Hq], x[:, Hq : Hq + Hkv], x[:, Hq + Hkv :]
    wq, wk = (weight(D, 2), weight(D, 3)) if norm else (None, None)
    tab = table(300, R) if R else torch.zeros(300, 0, device="cuda")
    rope = B.patch_rope(tab) if R else None
    pos = torch.randint(0, 300, (M,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(5))
    pages = (M + page - 1) // page + 2
    both = torch.full((pages, 2, Hkv, page, D), 3.0, dtype=BF, device="cuda")         # keys and values in one buffer, page by page
    cache = B.patch_kv_cache(both[:, 0], both[:, 1])
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(6))[:M].cuda()
    skip = slots.clone()
    skip[M // 2] = -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    qo = B.patch_kv_append(cache, k, v, skip, rope=rope, positions=pos if R else None, wk=wk, Q=q, wq=wq, status=status)
    want_q, want_k = B.patch_qk_norm_rope(q, k, rope, pos if R else None, wq=wq, wk=wk)
    want = torch.full_like(both, 3.0)
    for m in range(M):
        if int(skip[m]) >= 0:
            want[skip[m] // page, 0, :, skip[m] % page] = want_k[m]
            want[skip[m] // page, 1, :, skip[m] % page] = v[m]
    assert torch.equal(qo, want_q) and torch.equal(both, want) and int(status.item()) == 0
    # keys and values alone
    both.fill_(3.0)
    assert B.patch_kv_append(cache, k, v, skip, rope=rope, positions=pos if R else None, wk=wk) is None
    assert torch.equal(both, want)
    # a slot outside the cache is reported and not stored
    skip[0] = pages * page
    both.fill_(3.0)
    B.patch_kv_append(cache, k, v, skip, rope=rope, positions=pos if R else None, wk=wk, status=status)
    if int(slots[0]) >= 0 and M > 1:
        want[slots[0] // page, :, :, slots[0] % page] = 3.0
    else:
        want.fill_(3.0)
    assert torch.equal(both, want) and int(status.item()) == B.ERR_SIZE


def test_on_another_stream_and_in_a_graph(B):
    q = make(64, 8, 128, 1).contiguous()
    rope, pos, w = B.patch_rope(table(128, 128)), torch.arange(64, dtype=torch.int32, device="cuda"), weight(128, 2)
    want, _ = B.patch_qk_norm_rope(q, None, rope, pos, wq=w)
    s = torch.cuda.Stream()
    out = torch.zeros_like(q)
    s.wait_stream(torch.cuda.current_stream())
    B.patch_qk_norm_rope(q, None, rope, pos, wq=w, Q_out=out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.patch_qk_norm_rope(q, None, rope, pos, wq=w, Q_out=out)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("M", [64, 4096, 16384])
@pytest.mark.parametrize("weights", [False, True])
def test_a_gemm_behind_the_gradient(B, M, weights):
    """The gradient has completed when the next kernel starts: a GEMM whose weight and input are promised not to be written in its overlap
    window reads gQ without waiting, and one whose result is promised writes over an operand of the gradient."""
    H, D, N = 16, 128, 256
    g = torch.Generator(device="cuda").manual_seed(M)
    packed, layout = B.patch_pack((torch.randn(N, H * D, generator=g, device="cuda") * 0.05).to(BF), np.zeros((N // 128, H * D // 128), np.uint8))
    ws = torch.zeros(B.patch_gemm_workspace_size(layout, max(M, 64)), dtype=torch.uint8, device="cuda")
    q, gy = make(M, H, D, 1).contiguous(), make(M, H, D, 2).contiguous()
    w = weight(D, 3) if weights else None
    rope, pos = B.patch_rope(table(512, D)), (torch.arange(M, device="cuda") % 512).int()
    promised = B.VARIANT_AUTO | B.WEIGHTS_STATIC | B.INPUT_STATIC | (B.OUTPUT_STATIC if M <= 64 else 0)
    want, _, _, _ = B.patch_qk_norm_rope_backward(gy, None, rope, pos, Q=q, wq=w)
    torch.cuda.synchronize()
    want_y = B.patch_gemm(want.view(M, H * D), layout, packed, workspace=ws, variant=promised)
    torch.cuda.synchronize()
    gq, status = torch.empty_like(want), torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(8):
        gq.fill_(float("nan"))
        operand = gy.clone()                                    # the GEMM's result goes where the gradient's operand was
        y = operand.view(-1)[: M * N].view(M, N)
        B.patch_qk_norm_rope_backward(operand, None, rope, pos, Q=q, wq=w, gQ=gq, status=status)
        B.patch_gemm(gq.view(M, H * D), layout, packed, Y=y, workspace=ws, variant=promised)
        torch.cuda.synchronize()
        assert torch.equal(gq, want) and torch.equal(y, want_y) and int(status.item()) == 0


@pytest.mark.parametrize("case", [(9, 4, 2, 64, 32, True), (70, 6, 3, 128, 128, False), (33, 2, 5, 256, 64, False)])
def test_gradient_against_autograd(B, case):
    """The gradient kernel against torch's own differentiation of the definition in 64 bits."""
    M, Hq, Hkv, D, R, inter = case
    tab, pos = table(200, R), torch.randint(0, 200, (M,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(5))
    c, s = tab[pos.long(), : R // 2].double()[:, None], tab[pos.long(), R // 2 :].double()[:, None]
    rope = B.patch_rope(tab, interleaved=inter)
    ins = [make(M, Hq, D, 1), make(M, Hkv, D, 2), weight(D, 3), weight(D, 4)]
    gy = [make(M, Hq, D, 6), make(M, Hkv, D, 7)]
    got = B.patch_qk_norm_rope_backward(*gy, rope, pos, Q=ins[0], K=ins[1], wq=ins[2], wk=ins[3], eps=1e-5)
    leaves = [t.double().requires_grad_() for t in ins]
    loss = 0.0
    for x, w, g in zip(leaves[:2], leaves[2:], gy):
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5) * w
        a, b = (y[..., 0:R:2], y[..., 1:R:2]) if inter else (y[..., : R // 2], y[..., R // 2 : R])
        pair = (a * c - b * s, b * c + a * s)
        turned = torch.stack(pair, -1).flatten(-2) if inter else torch.cat(pair, -1)
        loss = loss + (torch.cat((turned, y[..., R:]), -1) * g.double()).sum()
    want = torch.autograd.grad(loss, leaves)
    for x, w, g, a, b in zip(ins, ins[2:], gy, got, want):
        x = x.double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
        most = 2 * g.double().abs().amax(-1, keepdim=True) * w.double().abs().max()
        check(a, b, r * (most + (x * r).abs() * most * (x * r).abs().mean(-1, keepdim=True)), "gradient")
    for x, g, a, b in zip(ins, gy, got[2:], want[2:]):
        xh = x.double() / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + 1e-5)
        assert bool(((a.double() - b).abs() <= (2 * g.double().abs().amax(-1, keepdim=True) * xh.abs()).sum((0, 1)) * 2.0 ** -12).all())
