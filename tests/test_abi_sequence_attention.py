"""Host-side checks of the attention within packed sequences: arguments refused before a device is touched."""
import ctypes

import pytest

FAKE = 1 << 20          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def B():
    from paper_2509_23410_b200 import build
    build.build()
    from paper_2509_23410_b200 import binding as b
    return b


SHAPES = (dict(M=-1), dict(M=2 ** 31 - 256), dict(B=-1), dict(B=(1 << 20) + 1), dict(D=32), dict(D=96), dict(D=256), dict(Hkv=0), dict(Hq=1), dict(Hq=7), dict(Hq=8192, Hkv=8192),
          dict(scale=0.0), dict(scale=-1.0), dict(scale=3e38), dict(scale=float("nan")), dict(scale=float("inf")), dict(ldq=1016), dict(ldq=1028), dict(ldk=248), dict(ldv=252),
          dict(ldo=0), dict(ldq=(1 << 28) + 8))


def test_forward_refusals(B):
    L = B.lib()

    def call(Q=FAKE, ldq=1024, K=FAKE, ldk=256, V=FAKE, ldv=256, M=100, Hq=8, Hkv=2, D=128, starts=FAKE, B=3, scale=0.1, O=FAKE, ldo=1024, lse=FAKE):
        return L.patch_sequence_attention(Q, ldq, K, ldk, V, ldv, M, Hq, Hkv, D, starts, B, scale, O, ldo, lse, None, None)
    assert call(M=0, Q=None, starts=None) == B.OK
    assert call(B=0, Q=None, starts=None) == B.OK
    for kw in SHAPES:
        assert call(**kw) == B.ERR_SHAPE, kw
    for kw in (dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(starts=None)):
        assert call(**kw) == B.ERR_NULL, kw
    for kw in (dict(Q=FAKE + 2), dict(K=FAKE + 8), dict(V=FAKE + 4), dict(O=FAKE + 8), dict(starts=FAKE + 2), dict(lse=FAKE + 1)):
        assert call(**kw) == B.ERR_ALIGN, kw


def test_backward_refusals(B):
    L = B.lib()
    need = B.patch_sequence_attention_backward_workspace_size(100, 3, 8, 2, 128)
    assert need > 0

    def call(gO=FAKE, ldgo=1024, Q=FAKE, ldq=1024, K=FAKE, ldk=256, V=FAKE, ldv=256, O=FAKE, ldo=1024, lse=FAKE, M=100, Hq=8, Hkv=2, D=128, starts=FAKE, B=3, scale=0.1,
             gQ=FAKE, ldgq=1024, gK=FAKE, ldgk=256, gV=FAKE, ldgv=256, ws=FAKE, wsb=need):
        return L.patch_sequence_attention_backward(gO, ldgo, Q, ldq, K, ldk, V, ldv, O, ldo, lse, M, Hq, Hkv, D, starts, B, scale, gQ, ldgq, gK, ldgk, gV, ldgv,
                                                   ws, wsb, None, None)
    assert call(M=0, Q=None, ws=None) == B.OK
    assert call(B=0, Q=None, ws=None) == B.OK
    for kw in SHAPES + (dict(ldgo=8), dict(ldgq=1000), dict(ldgk=260), dict(ldgv=0)):
        assert call(**kw) == B.ERR_SHAPE, kw
    for name in ("gO", "Q", "K", "V", "O", "lse", "starts", "gQ", "gK", "gV", "ws"):
        assert call(**{name: None}) == B.ERR_NULL, name
    for name in ("gO", "Q", "K", "V", "O", "gQ", "gK", "gV", "ws"):
        assert call(**{name: FAKE + 8}) == B.ERR_ALIGN, name
    assert call(ws=FAKE + 16) == B.ERR_ALIGN and call(lse=FAKE + 2) == B.ERR_ALIGN and call(starts=FAKE + 2) == B.ERR_ALIGN
    assert call(wsb=need - 1) == B.ERR_SIZE
    n = ctypes.c_size_t(0)
    assert L.patch_sequence_attention_backward_workspace_size(100, 3, 8, 2, 32, ctypes.byref(n)) == B.ERR_SHAPE
    assert L.patch_sequence_attention_backward_workspace_size(100, 3, 8, 2, 128, None) == B.ERR_NULL
