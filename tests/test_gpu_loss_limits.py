"""The largest and smallest calls from packed sequences to a loss; references and tolerances are those of test_gpu_logits and test_gpu_sequence_attention."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

from test_gpu_logits import B, check_distill, check_forward, logits, reference, special_rows, teacher  # noqa: E402, F401
from test_gpu_sequence_attention import Packed, run  # noqa: E402

MOST = 1 << 20


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M", [1, 3, 60])
def test_longest_rows(B, dtype, M):  # noqa: F811
    z = logits(M, MOST, dtype, 1)
    check_forward(B, z, 1.0, 256)
    check_forward(B, z, 0.5, 1)
    z[0] = 2.0                                                    # a border of 2^20 equal values
    check_forward(B, z, 1.0, 200)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("k", [100, 128, 129, 200, 256])
def test_most_alternatives_of_rows_of_one_cta(B, dtype, k):  # noqa: F811
    """As many rows as CTAs run, or more: each is one's alone, and its threads' bests are few for so many alternatives."""
    check_forward(B, logits(450, 70001, dtype, k), 1.0, k)
    check_forward(B, logits(900, 4099, dtype, k, 8), 1.0, k)
    z = torch.zeros(12 * 38, 20000, dtype=dtype, device="cuda")
    z.view(38, 12, 20000)[:] = special_rows(20000, dtype)
    check_forward(B, z, 1.0, k)
    z[:, 5000:] = 1.0                                             # thousands of equal ones, the border among them or above them
    check_forward(B, z, 1.0, k)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mask", ["-inf", "lowest"])
@pytest.mark.parametrize("M", [1, 13, 460])
def test_masked_rows_with_fewer_left_than_alternatives(B, dtype, mask, M):  # noqa: F811
    """A few columns are left of long rows, in one part of the row or in several; the others follow from the first column on."""
    V = 40011
    value = -math.inf if mask == "-inf" else torch.finfo(dtype).min
    full = logits(M, V, dtype, 9)
    for left in (1, 5, 30, 300):
        for where in (torch.randperm(V, device="cuda")[:left], torch.arange(V - left, V, device="cuda"), torch.arange(left, device="cuda") * 8 + 4096):
            z = torch.full((M, (V + 7) // 8 * 8), value, dtype=dtype, device="cuda")[:, :V]
            z[:, where] = full[:, where]
            for k in (1, 2, 20, 64, 256):
                check_forward(B, z, 1.0, k)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rest", [False, True])
def test_distill_of_longest_rows(B, dtype, rest):  # noqa: F811
    for M, K in ((1, 256), (40, 3)):
        z = logits(M, MOST, dtype, 2)
        ids, t = teacher(z, K, 1.0, 4, M, MOST)
        check_distill(B, z, ids, t, 1.0, rest, None, resident=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_short_rows(B, dtype):  # noqa: F811
    M, V = 300001, 9
    z = logits(M, V, dtype, 3)
    check_forward(B, z, 1.0, 2)
    ids, t = teacher(z, 2, 1.0, 4, M, V)
    check_distill(B, z, ids, t, 1.0, True, torch.linspace(-1, 1, M, device="cuda"))
    tokens = torch.arange(M, device="cuda") % V
    _, _, lse, _, _ = B.patch_token_logprobs(z, tokens, lse=True)
    gz = B.patch_token_logprobs_backward(z, tokens, lse, torch.ones(M, device="cuda"))
    want = torch.zeros(M, V, dtype=torch.float64, device="cuda").scatter_(1, tokens[:, None], 1.0) - reference(z, 1.0)[1]
    # p from lse of size up to 20: 2^-19 of it, and one rounding
    assert bool(((gz.double() - want).abs() <= 2.0 ** -18 + torch.finfo(dtype).eps / 2 * want.abs()).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1e-3, 40.0])
def test_cold_and_hot(B, dtype, T):  # noqa: F811
    M, V = 9, 5000
    z = logits(M, V, dtype, 5)
    check_forward(B, z, T, 30)
    ids, t = teacher(z, 16, T, 4, M, V)
    check_distill(B, z, ids, t, T, False, None)


@pytest.mark.parametrize("Hq,Hkv,lens", [(4096, 4096, [3, 2]), (4096, 1, [3, 2]), (64, 1, [1]), (64, 1, [300, 9]), (32, 1, [129] * 5)])
def test_most_heads(B, Hq, Hkv, lens):  # noqa: F811
    run(B, Packed(lens, Hq, Hkv, 64, seed=1))


def test_most_sequences(B):  # noqa: F811
    """2^20 sequences, almost all of them empty."""
    x = Packed([5, 130, 1], 2, 1, 64, seed=2)
    where = torch.zeros(MOST + 1, dtype=torch.int32, device="cuda")
    where[MOST // 3 :], where[MOST // 2 :], where[MOST - 1 :] = 5, 135, 136
    x.starts = where
    run(B, x)


def test_starts_that_cover_nothing(B):  # noqa: F811
    x = Packed([70], 2, 1, 64, seed=3)
    for starts in ([0, 0], [70, 70, 70], [35, 35]):
        o = torch.full((70, 2, 64), 5.0, dtype=BF, device="cuda")
        starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
        lse = torch.full((70, 2), 5.0, device="cuda")
        B.patch_sequence_attention(x.q, x.k, x.v, starts, O=o, lse=lse)
        g = [torch.full_like(y, 5.0) for y in (x.q, x.k, x.v)]
        B.patch_sequence_attention_backward(x.go, x.q, x.k, x.v, o, lse, starts, gQ=g[0], gK=g[1], gV=g[2])
        assert all(bool((y == 5.0).all()) for y in (o, lse, *g))
    assert math.isfinite(float(o.float().sum()))
