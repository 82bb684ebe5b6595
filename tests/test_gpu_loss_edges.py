"""Calls from packed sequences to a loss that the documentation allows at its edges: what lies beside a sequence, masked columns under large factors, temperatures and
logits of any size.  References and tolerances are those of test_gpu_logits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64

from test_gpu_logits import U, B, check, check_distill, check_forward, ln_tol, logits, reference, rounding, teacher  # noqa: E402, F401


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 40, 130, 300])
def test_rows_beside_a_sequence_leave_its_bits_alone(B, D, n):  # noqa: F811
    """The rows behind a sequence share tiles with its last ones; whatever they hold, results and gradients are the same bits.  Here their scores with the
    sequence's keys rise steeply, so that their maxima are raised again and again."""
    Hq, Hkv, M = 4, 2, 512
    g = torch.Generator(device="cuda").manual_seed(n)
    q, k, v, go = (torch.randn(M, h, D, generator=g, device="cuda").to(BF) for h in (Hq, Hkv, Hkv, Hq))
    k[:n] += torch.linspace(0, 2, n, device="cuda")[:, None, None].to(BF)
    got = []
    for other in (0.0, 1.0, 30.0, -30.0, math.nan):
        q[n:] = other
        for starts in ([0, n], [0, n, M]):
            where = torch.tensor(starts, dtype=torch.int32, device="cuda")
            lse = torch.zeros(M, Hq, device="cuda")
            o = B.patch_sequence_attention(q, k, v, where, O=torch.zeros_like(q), lse=lse)
            grads = B.patch_sequence_attention_backward(go, q, k, v, o, lse, where)
            got.append([x[:n].clone() for x in (o, lse, *grads)])
    for other in got[1:]:
        # (the gradients of keys are summed in as many parts as the number of sequences suggests: equal numbers of them are compared)
        assert all(torch.equal(a, b) for a, b in zip(got[0][:3], other[:3]))
    assert all(torch.equal(a, b) for first in (0, 1) for i in range(first, len(got), 2) for a, b in zip(got[first], got[i]))


@pytest.mark.parametrize("dtype,M,V", [(F32, 1400, 16384), (BF, 1400, 32768), (BF, 300, 131072)])
def test_listed_columns_do_not_show_in_the_rows_that_follow(B, dtype, M, V):  # noqa: F811
    """Rows in shared memory follow one another in the same places, where the listed columns of each are overwritten: other ones in every row, in whole blocks and
    spread.  All logits are equal, so that a -inf of another row would change a row's loss and gradient."""
    K = 256
    z = torch.ones(M, V, dtype=dtype, device="cuda")
    first = (torch.arange(M, device="cuda") * 7919) % (V - 16 * K)
    step = torch.where(torch.arange(M, device="cuda") % 2 == 0, 1, 16)
    ids = (first[:, None] + step[:, None] * torch.arange(K, device="cuda")).int()
    t = torch.full((M, K), math.log(0.5 / K), device="cuda")
    for _ in range(3):
        gz = torch.empty_like(z)
        loss = B.patch_distill_loss(z, ids, t, rest=True, gZ=gz)
        want = 0.5 * math.log(V) + 0.5 * math.log(V / (V - K))
        assert float((loss - want).abs().max()) < 1e-4
        assert len(loss.unique()) == 1                            # the same sums, whatever the list's columns
        out = 1.0 / V - 0.5 / (V - K)                             # p (1 - q_r / p_r) and p - q
        inside = torch.zeros(M, V, dtype=torch.bool, device="cuda").scatter_(1, ids.long(), True)
        assert float((gz.float()[~inside] / out - 1).abs().max()) < 2.0 ** -7 and float((gz.float()[inside] / (1.0 / V - 0.5 / K) - 1).abs().max()) < 2.0 ** -7


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [1.0, 1e6, 1e12])
def test_entropy_gradient_of_masked_columns_is_zero_whatever_its_factor(B, dtype, size):  # noqa: F811
    M, V, T = 5, 3001, 0.5
    z = logits(M, V, dtype, 8)
    z[:, 100:200], z[:, 200:300], z[2, 7:] = -math.inf, torch.finfo(dtype).min, -math.inf
    _, ent, lse, _, _ = B.patch_token_logprobs(z, temperature=T, entropy=True, lse=True)
    gent = torch.full((M,), size, device="cuda")
    gz = B.patch_token_logprobs_backward(z, None, lse, entropy=ent, gentropy=gent, temperature=T)
    assert bool((gz[:, 100:300] == 0).all()) and bool((gz[2, 7:] == 0).all())
    lnp, p, _, h = reference(z, T)
    want = torch.where(p > 0, -size / T * p * (torch.where(p > 0, lnp, 0.0) + h[:, None]), 0.0)
    rel = 4 * (ln_tol(z, V, T)[:, None] + 8 * U)
    check(gz, want, rel * size / T * p * (torch.where(p > 0, lnp, 0.0).abs() + math.log(V) + 1) + rounding(want, dtype, 1e-30 * size))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1e-6, 1e24, 1e30, 1e33])
@pytest.mark.parametrize("M,V", [(1, 40000), (700, 600)])
def test_logits_and_temperatures_of_any_size(B, dtype, T, M, V):  # noqa: F811
    """The distribution depends on z / T alone: rows of ordinary ratios at any scale, with columns masked by -inf and the type's lowest value."""
    z = logits(M, V, dtype, 9, scale=3.0 * T)
    z[0, 100:200] = -math.inf
    if T < 1e28:                                                  # else the lowest value is no mask
        z[0, 300:400] = torch.finfo(dtype).min
    check_forward(B, z, T, 7)
    ids, t = teacher(z, 12, T, 4, M, V)
    for rest in (False, True):
        check_distill(B, z, ids, t, T, rest, torch.full((M,), T, device="cuda"))        # the factor makes the gradients' size p again


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [50, 40000])
def test_masked_columns_that_are_asked_for(B, dtype, V):  # noqa: F811
    """A masked column has no gradient unless it is the token or listed: then the loss is infinite, and the gradient is the formula's."""
    M = 3
    z = logits(M, V, dtype, 5)
    z[:, 10:20] = -math.inf
    tokens = torch.tensor([12, 3, 19], device="cuda")
    logp, _, lse, _, _ = B.patch_token_logprobs(z, tokens, lse=True)
    assert logp[[0, 2]].tolist() == [-math.inf] * 2 and math.isfinite(float(logp[1]))
    glogp = torch.tensor([2.0, 2.0, 0.0], device="cuda")
    gz = B.patch_token_logprobs_backward(z, tokens, lse, glogp)
    assert float(gz[0, 12]) == 2.0 and bool((gz[0, [10, 11, 13, 19]] == 0).all()) and bool((gz[1, 10:20] == 0).all()) and bool((gz[2] == 0).all())
    ids = torch.tensor([[12, 3, -1], [3, 4, 5], [15, 15, 1]], dtype=torch.int32, device="cuda")
    t = torch.tensor([[-1.0, -2.0, 0.0], [-1.0, -2.0, -3.0], [-2.0, -1.0, -math.inf]], device="cuda")
    for rest in (False, True):
        q = t.double().exp() if rest else torch.softmax(t.double().masked_fill(ids < 0, -math.inf), -1)
        stats, fused = torch.empty(M, 2, device="cuda"), torch.empty(M, (V + 7) // 8 * 8, dtype=dtype, device="cuda")[:, :V]
        loss = B.patch_distill_loss(z, ids, t, rest=rest, stats=stats, gZ=fused)
        assert loss[[0, 2]].tolist() == [math.inf] * 2 and math.isfinite(float(loss[1]))
        for gz in (fused, B.patch_distill_loss_backward(z, ids, t, stats, rest=rest)):
            assert not bool(gz.isnan().any())
            want = torch.zeros(M, 10, dtype=F64, device="cuda")
            want[0, 2], want[2, 5] = -q[0, 0], -q[2, :2].sum()
            check(gz[:, 10:20], want, rounding(want, dtype) + 8 * U)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype,M", [(F32, 273), (BF, 452)])
def test_gradients_of_rows_whose_stores_are_slow(B, dtype, M, rest):  # noqa: F811
    """Rows in shared memory that fill their places there, and whose pitch is a large power of two: stores wait, and the copies of the rows that follow are not to
    overtake the last reading of a row."""
    V = 131072
    z = logits(M, V, dtype, 35)
    ids, t = teacher(z, 96, 0.7, 4, M, V)
    gloss = torch.randn(M, device="cuda")
    check_distill(B, z, ids, t, 0.7, rest, gloss, resident=True)
    got = []
    for _ in range(25):
        gz = torch.empty_like(z)
        B.patch_distill_loss(z, ids, t, temperature=0.7, rest=rest, gloss=gloss, gZ=gz)
        got = got[:1] + [gz]
        assert torch.equal(got[0], got[-1])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("T", [1.0, 50.0])
@pytest.mark.parametrize("M,V", [(12, 300), (12, 40000), (460, 20000)])
def test_students_masked_by_the_lowest_value(B, dtype, rest, T, M, V):  # noqa: F811
    """Columns masked by the type's lowest value: all but the listed ones, all but some of them, all of a row.  The gradient in a launch of its own is as exact as the one beside
    the loss."""
    K = 20
    z, low = logits(M, V, dtype, 6, scale=3.0 * T), torch.finfo(dtype).min
    ids, t = teacher(z, K, T, 4, M, V)
    own = torch.gather(z, 1, ids.long())
    z[1::5] = low
    z[1::5] = z[1::5].scatter(1, ids[1::5].long(), own[1::5])     # the listed ones are left
    z[2::5] = low
    z[2::5] = z[2::5].scatter(1, ids[2::5, : K // 2].long(), own[2::5, : K // 2])
    z[3::5] = low                                                 # nothing is: an even distribution
    z[4::5, : V // 2] = low
    gloss = torch.randn(M, device="cuda")
    # differences first: beside values of 3e38 even 64 bits leave nothing of a logarithm
    x, inside = z.to(F64), torch.zeros(M, V, dtype=torch.bool, device="cuda").scatter_(1, ids.long(), True)
    p = torch.softmax((x - x.amax(-1, keepdim=True)) / T, -1)
    q = t.to(F64).exp() if rest else torch.softmax(t.to(F64), -1)
    want, size = p - torch.zeros_like(p).scatter_(1, ids.long(), q), p + torch.zeros_like(p).scatter_(1, ids.long(), q)
    if rest:
        q_r = 1 - q.sum(-1, keepdim=True)
        out = x.masked_fill(inside, -math.inf)
        w = torch.softmax((out - out.amax(-1, keepdim=True)) / T, -1)
        p_r = p.masked_fill(inside, 0.0).sum(-1, keepdim=True)
        want, size = torch.where(inside, want, w * (p_r - q_r)), torch.where(inside, size, w * (p_r + q_r))
    g = gloss.to(F64)[:, None] / T
    stats, fused = torch.empty(M, 2, device="cuda"), torch.empty(M, (V + 7) // 8 * 8, dtype=dtype, device="cuda")[:, :V]
    loss = B.patch_distill_loss(z, ids, t, temperature=T, rest=rest, stats=stats, gloss=gloss, gZ=fused)
    assert not bool(loss.isnan().any())
    rel = 4 * (V / 512 + 64 + 3 * 60) * U + 300 * U               # as in check_distill, ordinary logits over T at most 15 in size
    left = (4 + K) * U * torch.where(inside, p, w) if rest else 0.0
    for gz in (fused, B.patch_distill_loss_backward(z, ids, t, stats, gloss=gloss, temperature=T, rest=rest)):
        check(gz, want * g, (rel * size + left) * g.abs() + rounding(want * g, dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rest", [False, True])
def test_gradient_in_a_launch_of_its_own_of_cold_rows(B, dtype, rest):  # noqa: F811
    """Logits of tens of thousands over the temperature: probabilities are as exact as beside the loss."""
    M, V, K, T = 7, 3001, 16, 1e-4
    z = logits(M, V, dtype, 5, scale=1e-4) + 8.0
    pad = torch.zeros(M, 3008, dtype=dtype, device="cuda")[:, :V]
    pad.copy_(z)
    if dtype is F32:
        pad += 1e-4 * torch.randn(M, V, device="cuda")
    ids, t = teacher(pad, K, T, 4, M, V)
    stats, fused = torch.empty(M, 2, device="cuda"), torch.empty(M, 3008, dtype=dtype, device="cuda")[:, :V]
    B.patch_distill_loss(pad, ids, t, temperature=T, rest=rest, stats=stats, gZ=fused)
    alone = B.patch_distill_loss_backward(pad, ids, t, stats, temperature=T, rest=rest)
    assert float((alone.double() - fused.double()).abs().max() * T) <= 2.0 ** -18 + (2.0 ** -8 if dtype is BF else 0.0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1.0, 0.7, 50.0, 1e-4])
@pytest.mark.parametrize("V", [9, 3000, 50257])
def test_gradient_of_rows_whose_lse_says_too_little(B, dtype, T, V):  # noqa: F811
    """Rows of nothing but the type's lowest value (an even distribution), cold ones, and ordinary ones and rows without a distribution among them; in place too."""
    M = 9
    z = logits(M, V, dtype, 6, extra=8)
    z[1::4], z[2::4, V // 2 :], z[3, :] = torch.finfo(dtype).min, torch.finfo(dtype).min, -math.inf
    z[6] = torch.finfo(dtype).max                                 # and of nothing but the highest
    g = torch.Generator(device="cuda").manual_seed(3)
    tokens = torch.randint(0, V // 2, (M,), generator=g, device="cuda")
    glogp, gent = (torch.randn(M, generator=g, device="cuda") for _ in range(2))
    glogp[4], gent[4], tokens[0] = 0.0, 0.0, -1
    _, ent, lse, _, _ = B.patch_token_logprobs(z, tokens, temperature=T, entropy=True, lse=True)
    x = z.to(F64)
    none = (x == -math.inf).all(-1, keepdim=True)
    x = (x - x.amax(-1, keepdim=True).clamp(min=-4e38)) / T       # differences first: beside 3e38 even 64 bits leave nothing of a logarithm
    lnp = torch.log_softmax(torch.where(none, 0.0, x), -1)
    p = torch.where(none, 0.0, lnp.exp())
    lnp = torch.where(p > 0, lnp, 0.0)
    hot = torch.zeros(M, V, dtype=F64, device="cuda").scatter_(1, tokens.clamp(min=0)[:, None], (tokens >= 0).to(F64)[:, None])
    hot = torch.where(none, 0.0, hot)
    a, h = torch.where(tokens >= 0, glogp, 0.0).to(F64)[:, None], -(p * lnp).sum(-1, keepdim=True)
    seen = lse.to(F64).abs().clamp(max=32768.0)[:, None] * 2.0 ** -23 + (V / 512 + 64) * U                 # beyond it nothing comes from lse
    for use in ("logp", "entropy", "both"):
        ga, ge = (a if use != "entropy" else 0 * a), (gent.to(F64)[:, None] if use != "logp" else 0 * a)
        want = (ga * (hot - p) - ge * p * (lnp + h)) / T
        size = (ga.abs() * p + ge.abs() * p * (lnp.abs() + h + 1)) / T
        kw = dict(temperature=T, **(dict(entropy=ent, gentropy=gent) if use != "logp" else {}))
        gl = glogp if use != "entropy" else None
        # logits of size 5 over T: the exponent's product is off by 2^-23 of itself, which is at most 110 where p is not 0
        tol = 2 * (seen + 110 * 2.0 ** -23) * size + (ga.abs() * hot / T) * 4 * U + rounding(want, dtype)
        gz = B.patch_token_logprobs_backward(z, tokens, lse, gl, **kw)
        check(gz, want, tol)
        same = torch.empty(M, (V + 7) // 8 * 8, dtype=dtype, device="cuda")[:, :V]
        same.copy_(z)
        B.patch_token_logprobs_backward(same, tokens, lse, gl, gZ=same, **kw)
        assert torch.equal(same, gz)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mask", [-math.inf, "lowest", -1e9])
@pytest.mark.parametrize("M,V,K", [(20, 300, 12), (20, 40000, 256), (460, 20000, 40)])
def test_lists_that_cover_all_that_a_mask_leaves(B, dtype, mask, M, V, K):  # noqa: F811
    """Teacher and student have the same few columns left, all of them listed: the rest is nothing, whatever rounding makes of the list's sum.  A rest that is
    more than rounding has no place: the loss is infinite."""
    z, full = logits(M, V, dtype, 6), logits(M, V, F32, 7)
    left = torch.rand(M, V, device="cuda").topk(K - 3, -1).indices
    keep = torch.zeros(M, V, dtype=torch.bool, device="cuda").scatter_(1, left, True)
    z[~keep], full[~keep] = torch.finfo(dtype).min if mask == "lowest" else mask, -math.inf
    *_, ids, t = B.patch_token_logprobs(full, k=K)                # the last three entries: probability 0
    gz = torch.empty(M, (V + 7) // 8 * 8, dtype=dtype, device="cuda")[:, :V]
    stats = torch.empty(M, 2, device="cuda")
    loss = B.patch_distill_loss(z, ids, t, rest=True, stats=stats, gZ=gz)
    q, lnp = t.to(F64).exp(), torch.log_softmax(z.to(F64), -1)
    want = -torch.where(q > 0, q * lnp.gather(1, ids.long()), 0.0).sum(-1)
    check(loss, want, 2 * ln_tol(z, V, 1.0) + 300 * U * want)
    p = lnp.exp()
    hot = torch.zeros_like(p).scatter_(1, ids.long(), q)
    for g in (gz, B.patch_distill_loss_backward(z, ids, t, stats, rest=True)):
        check(g, p - hot, 4 * (ln_tol(z, V, 1.0)[:, None] + 300 * U) * (p + hot) + rounding(p - hot, dtype))
    t[:, 0] -= 0.1
    loss = B.patch_distill_loss(z, ids, t, rest=True, gZ=gz)
    assert bool((loss > 1e4).all()) and not bool(gz.isnan().any()) and (mask != -math.inf or bool((loss == math.inf).all()))
