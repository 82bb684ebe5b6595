"""Host-side checks of the entry points from logits to a loss: arguments refused before a device is touched."""
import pytest

FAKE = 1 << 20          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def B():
    from paper_2509_23410_b200 import build
    build.build()
    from paper_2509_23410_b200 import binding as b
    return b


def refused(call, B, shape=(), null=(), align=()):
    for status, kws in ((B.ERR_SHAPE, shape), (B.ERR_NULL, null), (B.ERR_ALIGN, align)):
        for kw in kws:
            assert call(**kw) == status, kw


LOGITS = (dict(M=-1), dict(M=1 << 31), dict(V=0), dict(V=(1 << 20) + 1), dict(ldz=992), dict(ldz=1004), dict(ldz=1 << 61), dict(dtype=2), dict(dtype=-1),
          dict(T=0.0), dict(T=-1.0), dict(T=float("inf")), dict(T=float("nan")), dict(T=1e-42))


def test_logprobs_refusals(B):
    L = B.lib()

    def call(Z=FAKE, ldz=1000, dtype=0, M=4, V=1000, tokens=FAKE, k=5, T=1.0, logp=FAKE, ent=FAKE, lse=FAKE, ids=FAKE, top=FAKE):
        return L.patch_token_logprobs(Z, ldz, dtype, M, V, tokens, k, T, logp, ent, lse, ids, top, None, None)
    assert call(M=0, Z=None, tokens=None, logp=None) == B.OK
    refused(call, B, LOGITS + (dict(k=-1), dict(k=257), dict(V=4, k=5)),
            (dict(Z=None), dict(tokens=None), dict(logp=None), dict(ids=None), dict(top=None), dict(tokens=None, logp=None, ent=None, lse=None, k=0)),
            (dict(Z=FAKE + 8), dict(tokens=FAKE + 4), dict(logp=FAKE + 2), dict(ent=FAKE + 1), dict(lse=FAKE + 2), dict(ids=FAKE + 2), dict(top=FAKE + 2)))


def test_logprobs_backward_refusals(B):
    L = B.lib()

    def call(Z=FAKE, ldz=1000, dtype=1, M=4, V=1000, tokens=FAKE, T=1.0, lse=FAKE, glogp=FAKE, ent=FAKE, gent=FAKE, gZ=2 * FAKE, ldg=1000):
        return L.patch_token_logprobs_backward(Z, ldz, dtype, M, V, tokens, T, lse, glogp, ent, gent, gZ, ldg, None, None)
    assert call(M=0, Z=None, gZ=None) == B.OK
    refused(call, B, LOGITS + (dict(ldg=992), dict(ldg=1001), dict(gZ=FAKE, ldg=1008)),
            (dict(Z=None), dict(gZ=None), dict(lse=None), dict(glogp=None, gent=None), dict(tokens=None), dict(ent=None)),
            (dict(Z=FAKE + 8), dict(gZ=FAKE + 4), dict(tokens=FAKE + 4), dict(lse=FAKE + 2), dict(glogp=FAKE + 2), dict(ent=FAKE + 2), dict(gent=FAKE + 2)))


@pytest.mark.parametrize("flags", [0, 1])
def test_distill_refusals(B, flags):
    L = B.lib()

    def call(Z=FAKE, ldz=1000, dtype=0, M=4, V=1000, ids=FAKE, t=FAKE, K=8, T=1.0, flags=flags, loss=FAKE, stats=FAKE, gloss=FAKE, gZ=2 * FAKE, ldg=1000):
        return L.patch_distill_loss(Z, ldz, dtype, M, V, ids, t, K, T, flags, loss, stats, gloss, gZ, ldg, None, None)
    assert call(M=0, Z=None, ids=None, loss=None) == B.OK
    more = (dict(K=0), dict(K=257), dict(flags=2), dict(ldg=992), dict(ldg=1001))
    align = (dict(Z=FAKE + 8), dict(gZ=FAKE + 4), dict(ids=FAKE + 2), dict(t=FAKE + 2), dict(stats=FAKE + 2), dict(gloss=FAKE + 2))
    refused(call, B, LOGITS + more + (dict(gZ=FAKE, ldg=1008),), (dict(Z=None), dict(ids=None), dict(t=None), dict(loss=None)), align + (dict(loss=FAKE + 2),))

    def back(Z=FAKE, ldz=1000, dtype=0, M=4, V=1000, ids=FAKE, t=FAKE, K=8, T=1.0, flags=flags, stats=FAKE, gloss=FAKE, gZ=2 * FAKE, ldg=1000):
        return L.patch_distill_loss_backward(Z, ldz, dtype, M, V, ids, t, K, T, flags, stats, gloss, gZ, ldg, None, None)
    assert back(M=0, Z=None, ids=None) == B.OK
    refused(back, B, LOGITS + more + (dict(gZ=FAKE),), (dict(Z=None), dict(ids=None), dict(t=None), dict(stats=None), dict(gZ=None)), align)


def test_the_binding_refuses_what_is_not_on_the_gpu(B):
    torch = pytest.importorskip("torch")
    z = torch.zeros(2, 8)
    for call in (lambda: B.patch_token_logprobs(z, k=1, lse=torch.zeros(2), stream=S), lambda: B.patch_token_logprobs(z[0], k=1, stream=S),
                 lambda: B.patch_distill_loss(z, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1), loss=torch.zeros(2), stream=S),
                 lambda: B.patch_token_logprobs_backward(z, None, torch.zeros(2), gZ=z, stream=S),
                 lambda: B.patch_distill_loss_backward(z, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1), torch.zeros(2, 2), gZ=z, stream=S)):
        with pytest.raises(AssertionError):
            call()


class S:
    cuda_stream = 0
