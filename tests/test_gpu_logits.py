"""Log probabilities, entropy, top alternatives, their gradient, and distillation from a teacher's list, against the definitions in 64 bits.

Tolerances.  u = 2^-24.  A term 2^((x - m) c) is off by 4 u (the exponential instruction, two ulp) and u |ln p| (the exponent's product and
c, half an ulp each); weighted by p, that is at most (4 + 2 H) u with H <= ln V < 14: 32 u.  A thread adds up to V / 512 + 8 terms of one half of a pair (fewer
where CTAs share a row), then 13 sums join: in all (V / 512 + 64) u relative in S, the same absolute in ln S.  Division and subtraction add 2 u of the
results' size and of the largest logit over T.  The entropy's second sum is as exact relative to itself, H or less.
Gradients: p is off relatively by the error of lse plus 2 u |z / T| and the exponential's; products add 4 u; one rounding to the logits' type."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2509_23410_b200 import build, binding as b
    build.build()
    return b


def logits(M, V, dtype, seed, extra=0, scale=3.0):
    """[M, V] in a buffer of a larger pitch whose other columns are NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = (V + 7) // 8 * 8 + extra
    z = torch.full((M, ld), math.nan, device="cuda", dtype=dtype)
    z[:, :V] = (scale * torch.randn(M, V, generator=g, device="cuda")).to(dtype)
    return z[:, :V]


def special_rows(V, dtype):
    """Rows where things can go wrong; all but the last two have a distribution or none at all."""
    g = torch.Generator(device="cuda").manual_seed(V)
    r = (2 * torch.randn(12, V, generator=g, device="cuda")).to(dtype)
    i = torch.arange(V, device="cuda")
    r[0] = 1.5                                                    # all equal
    r[1] = -math.inf                                              # nothing
    r[2, 3:] = -math.inf                                          # three or fewer left
    r[3] = (i.float() * 0.001).to(dtype)                          # ascending
    r[4] = (-i.float() * 0.001).to(dtype)                         # descending
    r[5] = torch.where(i % 2 == 0, 0.0, -0.0).to(dtype)           # both zeros
    r[6] = torch.finfo(dtype).min                                 # the type's lowest value throughout
    r[7, i % 3 != 1] = torch.finfo(dtype).min                     # as a mask
    r[8, V // 2] = 300.0                                          # one certain token
    r[9, : V - 1] = -math.inf                                     # only the last one
    r[10] = torch.where(i % 256 == 7 % max(1, V), 5.0, -5.0).to(dtype)   # the best ones a thread apart
    r[11, : V // 2] = 4.0                                         # a border of many equal values
    return r


def reference(z, T):
    z = z.to(F64)
    x = z / T
    m = x.amax(-1, keepdim=True)
    none = m == -math.inf
    e = torch.where(none, 0.0, torch.exp(x - torch.where(none, 0.0, m)))
    s = e.sum(-1, keepdim=True)
    lse = torch.where(none, -math.inf, m + s.log())
    lnp = torch.where(none, -math.inf, x - lse)
    p = torch.where(none, 0.0, lnp.exp())
    return lnp, p, lse.squeeze(-1), -(p * torch.where(p > 0, lnp, 0.0)).sum(-1)


def ln_tol(z, V, T):
    top = torch.nan_to_num(z.to(F64).amax(-1).abs(), 0.0, 0.0, 0.0) / T
    return (V / 512 + 64) * U + 3 * U * (top + math.log(V) + 1)


def check(got, want, tol):
    got, want = got.to(F64), want.to(F64)
    same = (got == want) | (got.isnan() & want.isnan())
    ok = same | ((got - want).abs() <= tol)
    assert bool(ok.all()), float((got - want).abs()[~ok].max())


def order(z, k):
    z = torch.where(z.isnan(), -math.inf, z.to(F64))
    return torch.sort(z, stable=True, dim=-1, descending=True).indices[:, :k]


def check_forward(B, z, T, k, status=None):
    M, V = z.shape
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda")
    tokens[::5] = -1 - tokens[::5]
    logp, ent, lse, ids, top = B.patch_token_logprobs(z, tokens, k=k, temperature=T, entropy=True, lse=True)
    lnp, p, want_lse, want_ent = reference(z, T)
    tol = ln_tol(z, V, T)
    want = torch.where(tokens >= 0, lnp.gather(1, tokens.clamp(min=0)[:, None]).squeeze(1), 0.0)
    check(logp, want, tol + 3 * U * torch.nan_to_num(want.abs(), 0.0, 0.0, 0.0))
    check(lse, want_lse, tol)
    check(ent, want_ent, 2 * tol + (V / 512 + 64) * U * (want_ent + 1))
    if k:
        want_ids = order(z, k)
        assert bool((ids == want_ids).all())
        want = lnp.gather(1, want_ids)
        check(top, want, tol[:, None] + 3 * U * torch.nan_to_num(want.abs(), 0.0, 0.0, 0.0))
    else:
        assert ids is None and top is None


SIZES = [(1, 1, 0), (3, 2, 8), (2, 7, 0), (5, 8, 0), (4, 9, 16), (3, 255, 0), (2, 1000, 8), (7, 2049, 0), (1, 4096, 0), (2, 8192, 0), (1, 8193, 0),
         (700, 300, 0), (1, 32000, 0), (61, 50257, 24), (3, 128256, 0), (1, 151936, 8), (610, 5000, 0)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,V,extra", SIZES)
def test_logprobs(B, dtype, M, V, extra):
    for T, k in ((1.0, 0), (0.7, min(V, 1)), (2.0, min(V, 20)), (1.0, min(V, 256))):
        check_forward(B, logits(M, V, dtype, M + V, extra), T, k)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [1, 5, 300, 4099, 20000, 70001])
@pytest.mark.parametrize("k", [1, 17, 256])
def test_rows_of_equal_masked_and_extreme_values(B, dtype, V, k):
    z = special_rows(V, dtype)
    pad = torch.zeros(12, (V + 7) // 8 * 8, dtype=dtype, device="cuda")
    pad[:, :V] = z
    check_forward(B, pad[:, :V], 1.0, min(k, V))
    for r in (0, 2, 10):                                          # one row: by a cluster where it is long
        check_forward(B, pad[r : r + 1, :V], 1.5, min(k, V))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [300, 40000])
def test_nan_and_infinity_stay_in_their_rows(B, dtype, V):
    z = logits(6, V, dtype, 1)
    z[1, V // 3], z[3, V - 1], z[4] = math.nan, math.inf, math.nan
    clean = z.clone()
    clean[[1, 3, 4]] = 0.0
    tokens = torch.zeros(6, dtype=torch.int64, device="cuda")
    logp, ent, lse, ids, top = B.patch_token_logprobs(z, tokens, k=9, entropy=True, lse=True)
    lnp, p, want_lse, want_ent = reference(clean, 1.0)
    bad = torch.tensor([False, True, False, True, True, False], device="cuda")
    for got, want in ((logp, lnp[:, 0]), (lse, want_lse), (ent, want_ent)):
        assert bool(got[bad].isnan().all())
        check(got[~bad], want[~bad], 1e-4)
    assert bool((ids == order(z, 9)).all()) and bool(top[bad].isnan().all())
    gz = B.patch_token_logprobs_backward(z, tokens, lse, torch.ones(6, device="cuda"))
    assert bool(gz[bad].isnan().any(-1).all()) and not bool(gz[~bad].isnan().any())
    off = torch.where(bad, 0.0, 1.0).float()                      # rows that are not asked for: zeros, whatever they hold
    gz = B.patch_token_logprobs_backward(z, tokens, lse, off)
    assert not bool(gz.isnan().any()) and not bool(gz[bad].any())
    t_ids, t = torch.arange(4, dtype=torch.int32, device="cuda").repeat(6, 1), torch.full((6, 4), -1.5, device="cuda")
    for rest in (False, True):
        gz = torch.empty(6, (V + 7) // 8 * 8, dtype=dtype, device="cuda")[:, :V]
        loss = B.patch_distill_loss(z, t_ids, t, rest=rest, gloss=off, gZ=gz)
        assert bool(loss[bad].isnan().all()) and not bool(loss[~bad].isnan().any())
        assert not bool(gz.isnan().any()) and not bool(gz[bad].any())


def rounding(want, dtype, tiny=1e-30):
    """Half a step of the logits' type (values below its normal range: of the smallest normal)."""
    return torch.finfo(dtype).eps / 2 * want.abs() + tiny


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,V,extra", [(1, 1, 0), (3, 9, 16), (5, 300, 0), (2, 2049, 0), (61, 20000, 8), (3, 50257, 0)])
@pytest.mark.parametrize("use", ["logp", "entropy", "both"])
def test_logprobs_gradient(B, dtype, M, V, extra, use):
    T = 0.8
    z = logits(M, V, dtype, 7, extra)
    if V > 20:
        z[0, 5:15] = -math.inf
    g = torch.Generator(device="cuda").manual_seed(6)
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda")
    if M > 2:
        tokens[1] = -7
    glogp, gent = (torch.randn(M, generator=g, device="cuda") for _ in range(2))
    _, ent, lse, _, _ = B.patch_token_logprobs(z, tokens, temperature=T, entropy=True, lse=True)
    if use == "logp":
        gent = ent = None
    if use == "entropy":
        glogp = None
    gz = B.patch_token_logprobs_backward(z, tokens, lse, glogp, entropy=ent, gentropy=gent, temperature=T)
    leaf = torch.where(z.isinf(), -1e9, z.to(F64)).requires_grad_()        # differentiation of the definition (a mask far below, for its backward pass)
    lnp = torch.log_softmax(leaf / T, -1)
    f = leaf.sum() * 0
    if glogp is not None:
        f = f + (torch.where(tokens >= 0, lnp.gather(1, tokens.clamp(min=0)[:, None]).squeeze(1), 0.0) * glogp).sum()
    if gent is not None:
        f = f - ((lnp.exp() * lnp).sum(-1) * gent).sum()
    want, = torch.autograd.grad(f, leaf)
    p, size = lnp.detach().exp(), torch.zeros(M, 1, device="cuda", dtype=F64)
    rel = (V / 512 + 64) * U + 3 * U * (z.to(F64).abs().nan_to_num(0, 0, 0).amax(-1, keepdim=True) / T * 2 + math.log(V) + 1) + 8 * U
    if glogp is not None:
        size = size + glogp.abs()[:, None] / T * (p + (torch.arange(V, device="cuda") == tokens[:, None]))
    if gent is not None:
        size = size + gent.abs()[:, None] / T * p * (lnp.detach().abs() + math.log(V) + 1)
    check(gz, want, 4 * rel * size + rounding(want, dtype))
    inplace = z.clone() if V % 8 == 0 else logits(M, V, dtype, 7, 0)
    inplace.copy_(z)
    B.patch_token_logprobs_backward(inplace, tokens, lse, glogp, entropy=ent, gentropy=gent, temperature=T, gZ=inplace)
    assert torch.equal(inplace, gz)


def teacher(z, K, T, seed, M, V):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.nan_to_num(z.to(F64), 0.0, 0.0, -1e4) / T + torch.randn(M, V, generator=g, device="cuda")
    top, ids = torch.log_softmax(x, -1).topk(K, -1)
    return ids.to(torch.int32), top.float()


def distill_reference(z, ids, t, T, rest):
    """Losses [M], gradients of their sum, sizes of what is subtracted, and how the two change with q_r, what the list leaves; by the definition, entries
    that name one column added up."""
    lnp, p, lse, _ = reference(z, T)
    M, V = z.shape
    t, there = t.to(F64), (ids >= 0) & (ids < V)
    at = torch.where(there, ids, 0).long()
    q = torch.where(there, t.exp(), 0.0) if rest else torch.where(there, t, -math.inf)
    if not rest:
        q = torch.nan_to_num(torch.softmax(q, -1), 0.0)
    listed = torch.zeros(M, V, dtype=F64, device="cuda").scatter_add_(1, at, q)
    inside = torch.zeros(M, V, dtype=F64, device="cuda").scatter_add_(1, at, there.to(F64)) > 0
    loss = -torch.where(q > 0, q * lnp.gather(1, at), 0.0).sum(-1)
    total = q.sum(-1, keepdim=True)
    if not rest:
        return loss, torch.where(lse[:, None] == -math.inf, 0.0, p * total - listed), p * total + listed, (0.0, 0.0)          # no distribution: no gradient
    q_r = (1 - total).clamp(min=0)
    out = torch.where(inside, -math.inf, lnp)
    ln_r = torch.where((out == -math.inf).all(-1, keepdim=True), -math.inf, torch.logsumexp(torch.where((out == -math.inf).all(-1, keepdim=True), 0.0, out), -1, keepdim=True))
    loss = loss - torch.where(q_r > 0, q_r * ln_r, 0.0).squeeze(-1)
    w = torch.where(inside | (ln_r == -math.inf), 0.0, (lnp - ln_r).exp())
    none = lse[:, None] == -math.inf
    gz = torch.where(none, 0.0, torch.where(inside, p * (total + q_r) - listed, w * ((total + q_r) * ln_r.exp() - q_r)))
    change = torch.where(ln_r == -math.inf, 0.0, ln_r.abs()).squeeze(-1), torch.where(inside, p, w)
    return loss, gz, torch.where(inside, p + listed, w * (ln_r.exp() + q_r)), change


def check_distill(B, z, ids, t, T, rest, gloss, resident=False):
    M, V = z.shape
    loss = torch.empty(M, device="cuda")
    want_loss, want, size, change = distill_reference(z, ids, t, T, rest)
    # q_r = 1 - sum q in fp32: an exponential is off by up to 2 steps, 2^-22 of itself, each of K additions by 2^-24 of a sum of at most about 1; where the
    # list leaves next to nothing this is no small part of q_r, which enters the loss with ln p_r and the gradient with p or w
    left = (4 + ids.shape[1]) * U * 1.01
    tol = 2 * ln_tol(z, V, T) + 300 * U * torch.nan_to_num(want_loss.abs(), 0.0, 0.0, 0.0)        # up to 256 terms added
    tol = tol + left * change[0]
    g = gloss.to(F64)[:, None] / T if gloss is not None else 1.0 / T
    rel = 4 * ((V / 512 + 64) * U + 3 * U * (z.to(F64).abs().nan_to_num(0, 0, 0).amax(-1, keepdim=True).clamp(max=1e4) / T * 2 + math.log(V) + 1)) + 300 * U
    pitch = (V + 7) // 8 * 8
    buffers = [torch.full((M, pitch), 7.0, dtype=z.dtype, device="cuda") for _ in range(2)]
    stats = torch.empty(M, 2, device="cuda")
    B.patch_distill_loss(z, ids, t, temperature=T, rest=rest, loss=loss, stats=stats, gloss=gloss, gZ=buffers[0][:, :V])
    check(loss, want_loss, tol)
    alone = B.patch_distill_loss(z, ids, t, temperature=T, rest=rest)
    if resident:                                                  # another kernel than the loss alone
        check(alone, want_loss, tol)
    else:
        assert torch.equal(alone.nan_to_num(7.0), loss.nan_to_num(7.0))
    B.patch_distill_loss_backward(z, ids, t, stats, gloss=gloss, temperature=T, rest=rest, gZ=buffers[1][:, :V])
    for b in buffers:
        check(b[:, :V], want * g, (rel * size + left * change[1]) * (g.abs() if gloss is not None else g) + rounding(want * g, z.dtype))
        assert bool((b[:, V:] == 7.0).all()), "columns behind the vocabulary"
    same = torch.full((M, pitch), 7.0, dtype=z.dtype, device="cuda")[:, :V]
    same.copy_(z)
    B.patch_distill_loss(same, ids, t, temperature=T, rest=rest, gloss=gloss, gZ=same)
    assert torch.equal(same, buffers[0][:, :V])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("M,V,K,extra", [(1, 1, 1, 0), (3, 9, 4, 8), (5, 300, 256, 0), (2, 2049, 1, 0), (1, 32000, 32, 0), (61, 20001, 100, 0), (700, 600, 7, 0), (3, 70001, 64, 8)])
def test_distill(B, dtype, rest, M, V, K, extra):
    z = logits(M, V, dtype, 3, extra)
    ids, t = teacher(z, K, 1.5, 4, M, V)
    gloss = torch.randn(M, device="cuda")
    gloss[M // 2] = 0.0
    check_distill(B, z, ids, t, 1.5, rest, gloss if M > 1 else None)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("V", [40, 30000])
def test_distill_lists_with_gaps_repetitions_and_masked_students(B, dtype, rest, V):
    M, K = 9, 12
    z = logits(M, V, dtype, 3)
    ids, t = teacher(z, K, 1.0, 4, M, V)
    ids[0] = -1                                                   # no entry
    ids[1, 3:9] = -5                                              # gaps
    ids[2, 4:] = ids[2, 0]                                        # one column many times
    t[3, 2:6] = -math.inf                                         # probability 0
    t[4] = t[4] - 30                                              # a list that says next to nothing
    z[5, 20:] = -math.inf                                         # a masked student; listed columns among them
    z[6] = -math.inf                                              # nothing left of the student
    z[7, ids[7].long()] = 200.0                                   # all probability is listed
    z[8, ids[8].long()] = -200.0                                  # none is
    check_distill(B, z, ids, t, 1.0, rest, torch.linspace(-1, 2, M, device="cuda"))


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype,M,V,K", [(F32, 200, 32000, 9), (F32, 210, 32001, 1), (BF, 150, 98303, 64), (BF, 150, 98311, 40), (BF, 149, 128256, 256), (F32, 60, 128257, 33),
                                         (F32, 40, 200003, 12), (BF, 2000, 8000, 5)])
def test_distill_of_rows_that_stay_in_shared_memory(B, dtype, rest, M, V, K):
    """Batches whose rows in flight are more than L2 keeps: 1, 2, 4 and 8 CTAs to a row (and a batch just below, of short rows)."""
    z = logits(M, V, dtype, 3, 8)
    ids, t = teacher(z, K, 0.9, 4, M, V)
    ids[1], ids[2, K // 2 :] = -1, ids[2, :1]
    z[3, V // 3 :], z[4], z[5, ids[5].long()] = -math.inf, -math.inf, 150.0
    ids[6, 0], z[6, V - 1] = V - 1, 3.0                           # the last column, in the row's short vector where it has one
    z[7, V - 1] = 50.0
    gloss = torch.randn(M, device="cuda")
    gloss[M // 2] = 0.0
    check_distill(B, z, ids, t, 0.9, rest, gloss, resident=True)
    bad = z.clone() if V % 8 == 0 else z
    bad[9, V // 2], bad[M - 1, 0] = math.nan, math.inf
    gz = torch.zeros(M, (V + 7) // 8 * 8, dtype=dtype, device="cuda")[:, :V]
    loss = B.patch_distill_loss(bad, ids, t, temperature=0.9, rest=rest, gZ=gz)
    nan = torch.zeros(M, dtype=torch.bool, device="cuda")
    nan[[9, M - 1]] = True
    assert bool(loss[nan].isnan().all()) and bool(gz[nan].isnan().any(-1).all())
    assert not bool(loss[~nan].isnan().any()) and not bool(gz[~nan].isnan().any())


def test_everything_listed(B):
    """With the rest as a class and a list of all columns nothing is left for it."""
    z = logits(4, 24, F32, 1)
    ids = torch.stack([torch.randperm(24, device="cuda") for _ in range(4)]).int()
    t = torch.log_softmax(torch.randn(4, 24, device="cuda", dtype=F64), -1).float() + 1e-4         # sums to a little more than 1
    check_distill(B, z, ids, t, 1.0, True, None)


def test_one_entry_is_the_cross_entropy(B):
    z = logits(50, 32000, F32, 2)
    tokens = torch.randint(0, 32000, (50,), device="cuda")
    logp, _, lse, _, _ = B.patch_token_logprobs(z, tokens, lse=True)
    gz = torch.empty_like(z)
    loss = B.patch_distill_loss(z, tokens[:, None].int(), torch.zeros(50, 1, device="cuda"), gZ=gz)
    check(loss, -logp, 8 * U * (1 + logp.abs()))
    check(gz, B.patch_token_logprobs_backward(z, tokens, lse, torch.full((50,), -1.0, device="cuda")).to(F64), 64 * U)


def test_gradients_against_differences(B):
    """The loss's change along a direction, fp32 logits of a small vocabulary."""
    V, K, h = 64, 6, 2.0 ** -6
    z = logits(8, V, F32, 11, scale=1.0)
    ids, t = teacher(z, K, 1.0, 12, 8, V)
    d = torch.randn(8, V, device="cuda").round().clamp(-1, 1)
    for rest in (False, True):
        f = lambda x: B.patch_distill_loss(x.contiguous(), ids, t, rest=rest).double()  # noqa: E731
        gz = torch.empty_like(z)
        B.patch_distill_loss(z, ids, t, rest=rest, gZ=gz)
        # third derivatives of a cross entropy along d are at most 2 |d|^3 = 2: h^2 / 6 * 2, and the losses' rounding over 2 h
        check((f(z + h * d) - f(z - h * d)) / (2 * h), (gz.double() * d).sum(-1), h * h / 3 + 200 * U * 8 / h)


def test_tokens_and_ids_out_of_range_are_reported(B):
    z, status = logits(3, 300, BF, 1), torch.zeros(1, dtype=torch.int32, device="cuda")
    tokens = torch.tensor([5, 300, 1 << 40], device="cuda")
    logp, _, lse, _, _ = B.patch_token_logprobs(z, tokens, lse=True, status=status)
    assert int(status) == B.ERR_SIZE and float(logp[0]) < 0 and not bool(logp[1:].any())
    status.zero_()
    gz = B.patch_token_logprobs_backward(z, tokens, lse, torch.ones(3, device="cuda"), status=status)
    assert int(status) == B.ERR_SIZE and not bool(gz[1:].any())
    ids, t = torch.tensor([[1, 2], [300, 3], [2 ** 31 - 1, 300]], dtype=torch.int32, device="cuda"), torch.full((3, 2), -1.0, device="cuda")
    for rest in (False, True):
        status.zero_()
        stats = torch.empty(3, 2, device="cuda")
        loss = B.patch_distill_loss(z, ids, t, rest=rest, status=status, stats=stats)
        assert int(status) == B.ERR_SIZE
        check(loss, distill_reference(z, ids, t, 1.0, rest)[0], 1e-4)
        status.zero_()
        B.patch_distill_loss_backward(z, ids, t, stats, rest=rest, status=status)
        assert int(status) == B.ERR_SIZE


@pytest.mark.parametrize("M,V", [(1, 128256), (40, 20000), (700, 5000)])
def test_equal_calls_give_equal_bits(B, M, V):
    z = logits(M, V, BF, 9)
    ids, t = teacher(z, 30, 1.0, 4, M, V)
    first = None
    for _ in range(3):
        gz = torch.empty_like(z)
        now = [x for x in B.patch_token_logprobs(z, ids[:, 0].long(), k=40, entropy=True, lse=True)] + [B.patch_distill_loss(z, ids, t, rest=True, gZ=gz), gz]
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


def test_captured_calls_follow_their_inputs_and_streams(B):
    z, other = logits(5, 20000, BF, 1), logits(5, 20000, BF, 2)
    ids, t = teacher(z, 8, 1.0, 4, 5, 20000)
    gz, loss, side = torch.empty_like(z), torch.empty(5, device="cuda"), torch.cuda.Stream()
    outs = [torch.empty(5, device="cuda"), torch.empty(5, 8, dtype=torch.int32, device="cuda"), torch.empty(5, 8, device="cuda")]

    def step():
        B.patch_token_logprobs(z, k=8, entropy=outs[0], top_ids=outs[1], top_logp=outs[2])
        B.patch_distill_loss(z, outs[1], outs[2], rest=True, loss=loss, gZ=gz)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    z.copy_(other)
    graph.replay()
    got = [x.clone() for x in (*outs, loss, gz)]
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, (*outs, loss, gz)))
    assert bool((outs[1] == order(other, 8)).all())
    # the student is its own teacher: the gradient vanishes but for rounding
    assert float(gz.abs().max()) < 1e-5


def test_offsets_beyond_32_bits(B):
    """Rows whose elements and bytes are numbered beyond 2^32."""
    M, ld, V = 34000, 131072, 500
    free, _ = torch.cuda.mem_get_info()
    if free < M * ld * 2 + (4 << 30):
        pytest.skip("needs 9 GB")
    z = torch.empty(M, ld, dtype=BF, device="cuda")[:, :V]
    z.copy_(logits(M, V, BF, 3))
    at = torch.tensor([0, 16383, 16384, 32768, M - 1], device="cuda")
    logp, ent, lse, ids, top = B.patch_token_logprobs(z, k=5, lse=True)
    check(lse[at], reference(z[at], 1.0)[2], 1e-4)
    assert bool((ids[at] == order(z[at], 5)).all())
    want_loss, want, size, _ = distill_reference(z[at], ids[at], top[at], 1.0, True)
    loss = B.patch_distill_loss(z, ids, top, rest=True, gZ=z)
    check(loss[at], want_loss, 1e-4)
    check(z[at], want, rounding(want, BF) + 1e-4 * size)


def test_refusals_of_the_binding(B):
    z = logits(4, 100, BF, 1)
    with pytest.raises(AssertionError):
        B.patch_token_logprobs(z.half(), k=1)
    with pytest.raises(AssertionError):
        B.patch_token_logprobs(z.t(), k=1)
    with pytest.raises(B.PatchError):
        B.patch_token_logprobs(torch.zeros(4, 100, dtype=BF, device="cuda"), k=1)         # a pitch of 100
    with pytest.raises(AssertionError):
        B.patch_token_logprobs(z, torch.zeros(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(AssertionError):
        B.patch_token_logprobs(z, k=3, top_ids=torch.zeros(4, 2, dtype=torch.int32, device="cuda"))
    with pytest.raises(B.PatchError):
        B.patch_token_logprobs(z, k=101)
    with pytest.raises(AssertionError):
        B.patch_distill_loss(z, torch.zeros(4, 2, device="cuda"), torch.zeros(4, 2, device="cuda"))
    with pytest.raises(AssertionError):
        B.patch_distill_loss(z, torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda"), gZ=z.float())
    with pytest.raises(B.PatchError):
        B.patch_distill_loss_backward(z, torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.zeros(4, 2, device="cuda"), gZ=z)
