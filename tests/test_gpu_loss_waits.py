"""Bounded waits of the kernels from packed sequences to a loss (and of the block kernel behind a prefix), made to run out in the test build (waits of 300 us; a status word tells CTA 0 to announce sixteen
bytes more than its first stage will ever receive).  Every role of the CTA has to find its end, and so have the CTAs that wait for it: the launch is reported and ends, and the
next one is as if nothing had been.  Nothing faults, traps or spins for ever."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

from test_gpu_logits import B, logits, teacher  # noqa: E402, F401
from test_gpu_sequence_attention import Packed  # noqa: E402

INJECT_MAGIC = 0x7E57


@pytest.fixture(scope="module")
def fi(B):  # noqa: F811
    from paper_2509_23410_b200 import build
    return B.load(build.build(fault_injection=True))


def ptr(t):
    return ctypes.c_void_p(t.data_ptr() if t is not None else 0)


def here():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype,M,V", [(F32, 1000, 16000), (F32, 1000, 32003), (BF, 450, 128256), (F32, 200, 128256), (F32, 50, 128256)])
def test_distillation_of_rows_in_shared_memory(B, fi, dtype, M, V, rest):  # noqa: F811
    """Rows of 1, 2, 4 and 8 CTAs, with several rows to a cluster and with one: the parts of a row wait for one another's sums."""
    K = 40
    z = logits(M, V, dtype, 3)
    ids, t = teacher(z, K, 1.0, 4, M, V)

    def call(lib, status):
        loss, gz = torch.zeros(M, device="cuda"), torch.zeros(M, (V + 7) // 8 * 8, dtype=dtype, device="cuda")
        rc = lib.patch_distill_loss(ptr(z), z.stride(0), B.LOGITS_F32 if dtype is F32 else B.LOGITS_BF16, M, V, ptr(ids), ptr(t), K, 1.0,
                                    B.DISTILL_REST if rest else 0, ptr(loss), None, None, ptr(gz), gz.stride(0), ptr(status), here())
        assert rc == B.OK
        torch.cuda.synchronize()
        return loss, gz, int(status)
    word = lambda v: torch.full((1,), v, dtype=torch.int32, device="cuda")  # noqa: E731
    want = call(B.lib(), word(0))
    assert want[2] == B.OK
    for _ in range(2):
        got = call(fi, word(0))
        assert got[2] == B.OK and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert call(fi, word(INJECT_MAGIC))[2] == B.ERR_TIMEOUT
    got = call(B.lib(), word(0))
    assert got[2] == B.OK and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,Hq,Hkv", [([1], 1, 1), ([90, 40], 2, 1), ([700, 300, 65], 4, 2), ([513, 128, 128, 300], 32, 32), ([300, 200], 48, 3)])
def test_attention_within_sequences(B, fi, D, lens, Hq, Hkv):  # noqa: F811
    """The forward kernel and both of the gradient; the first tile is a whole one, or one that is mended behind the sequence's end."""
    x = Packed(lens, Hq, Hkv, D, seed=1)
    M, n = x.M, len(lens)
    need = B.patch_sequence_attention_backward_workspace_size(M, n, Hq, Hkv, D)
    ld, ldo = x.q.stride(0), Hq * D
    word = lambda v: torch.full((1,), v, dtype=torch.int32, device="cuda")  # noqa: E731

    def forward(lib, status):
        o, lse = torch.zeros(M, Hq, D, dtype=BF, device="cuda"), torch.zeros(M, Hq, device="cuda")
        rc = lib.patch_sequence_attention(ptr(x.q), ld, ptr(x.k), ld, ptr(x.v), ld, M, Hq, Hkv, D, ptr(x.starts), n, D ** -0.5, ptr(o), ldo, ptr(lse), ptr(status),
                                          here())
        assert rc == B.OK
        torch.cuda.synchronize()
        return int(status), o, lse

    def backward(lib, status, o, lse):
        g = [torch.zeros(M, h, D, dtype=BF, device="cuda") for h in (Hq, Hkv, Hkv)]
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        rc = lib.patch_sequence_attention_backward(ptr(x.go), x.go.stride(0), ptr(x.q), ld, ptr(x.k), ld, ptr(x.v), ld, ptr(o), ldo, ptr(lse), M, Hq, Hkv, D, ptr(x.starts), n,
                                                   D ** -0.5, ptr(g[0]), ldo, ptr(g[1]), Hkv * D, ptr(g[2]), Hkv * D, ptr(ws), ws.numel(), ptr(status), here())
        assert rc == B.OK
        torch.cuda.synchronize()
        return int(status), *g
    want = forward(B.lib(), word(0))
    grads = backward(B.lib(), word(0), *want[1:])
    same = lambda a, b: a[0] == b[0] == B.OK and all(torch.equal(u, v) for u, v in zip(a[1:], b[1:]))  # noqa: E731
    for _ in range(2):
        assert same(forward(fi, word(0)), want)
        assert forward(fi, word(INJECT_MAGIC))[0] == B.ERR_TIMEOUT
        assert same(backward(fi, word(0), *want[1:]), grads)
        for kernel in (0, 1):                                     # of the queries, of the keys
            assert backward(fi, word(INJECT_MAGIC + kernel), *want[1:])[0] == B.ERR_TIMEOUT
    assert same(forward(B.lib(), word(0)), want) and same(backward(B.lib(), word(0), *want[1:]), grads)


@pytest.mark.parametrize("P", [120000, 262000])
def test_attention_behind_a_long_prefix(B, P):  # noqa: F811
    """The kernel that shares the way of a tile with them, with more tiles to a CTA than its ring holds."""
    import test_gpu_attention_limits as limits
    limits.test_a_wait_that_runs_out_is_reported_and_survivable(B, (40, 4, 1, P), 10000)
