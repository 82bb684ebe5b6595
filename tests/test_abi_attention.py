"""Host-side checks of the attention-side entry points: struct layouts, and arguments refused before a device is touched."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def B():
    from paper_2509_23410_b200 import build
    build.build()
    from paper_2509_23410_b200 import binding as b
    return b


def test_structs_match_header(B, tmp_path):
    for cls, name in ((B.Rope, "patch_rope_t"), (B.KVCache, "patch_kv_cache_t")):
        fields = [f for f, _ in cls._fields_]
        src = tmp_path / (name + ".c")
        src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "patch.h"\nint main(void) {\n'
                       f'  printf("%zu", sizeof({name}));\n' + "".join(f'  printf(" %zu", offsetof({name}, {f}));\n' for f in fields)
                       + "  return 0; }\n")
        exe = tmp_path / name
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
        got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
        assert got == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields]


def cache(B, **kw):
    a = dict(k_dev=FAKE, v_dev=FAKE, num_pages=10, page_stride=2 * 16 * 128, page_size=16, Hkv=2, D=128, reserved=0)
    a.update(kw)
    return B.KVCache(**a)


BAD_CACHES = [(dict(k_dev=None), "ERR_NULL"), (dict(v_dev=None), "ERR_NULL"), (dict(k_dev=FAKE + 2), "ERR_ALIGN"), (dict(v_dev=FAKE + 8), "ERR_ALIGN"),
              (dict(num_pages=0), "ERR_SHAPE"), (dict(num_pages=1 << 40), "ERR_SHAPE"), (dict(page_stride=2 * 16 * 128 - 8), "ERR_SHAPE"),
              (dict(page_stride=2 * 16 * 128 + 4), "ERR_SHAPE"), (dict(page_stride=1 << 62), "ERR_SHAPE"), (dict(page_size=8), "ERR_SHAPE"),
              (dict(page_size=24), "ERR_SHAPE"), (dict(page_size=512), "ERR_SHAPE"), (dict(Hkv=0), "ERR_SHAPE"), (dict(D=12), "ERR_SHAPE"),
              (dict(D=264), "ERR_SHAPE"), (dict(reserved=1), "ERR_SHAPE")]


def rope(B, **kw):
    a = dict(cos_sin_dev=FAKE, max_positions=64, rotary_dim=128, interleaved=0)
    a.update(kw)
    return B.Rope(**a)


BAD_ROPES = [(dict(cos_sin_dev=None), "ERR_NULL"), (dict(cos_sin_dev=FAKE + 4), "ERR_ALIGN"), (dict(max_positions=0), "ERR_SHAPE"),
             (dict(rotary_dim=144), "ERR_SHAPE"), (dict(rotary_dim=-16), "ERR_SHAPE"), (dict(rotary_dim=20), "ERR_SHAPE"),
             (dict(rotary_dim=12, interleaved=1), "ERR_SHAPE")]


def test_norm_rope_refusals(B):
    L = B.lib()

    def call(Q=FAKE, ldq=1024, Hq=8, K=FAKE, ldk=256, Hkv=2, M=4, D=128, wq=FAKE, wk=FAKE, r=rope(B), pos=FAKE, Qo=FAKE, ldqo=1024, Ko=FAKE, ldko=256):
        return L.patch_qk_norm_rope(Q, ldq, Hq, K, ldk, Hkv, M, D, wq, wk, 1e-6, r, pos, Qo, ldqo, Ko, ldko, None, None)
    assert call(M=0, Q=None, K=None) == B.OK
    assert call(Hq=0, Hkv=0) == B.OK
    for kw in (dict(M=-1), dict(D=4), dict(D=132), dict(D=264), dict(Hq=-1), dict(Hkv=1 << 20), dict(ldq=1016), dict(ldk=252), dict(ldqo=1028), dict(ldko=0)):
        assert call(**kw) == B.ERR_SHAPE, kw
    for kw in (dict(Q=None), dict(K=None), dict(Qo=None), dict(Ko=None), dict(pos=None)):
        assert call(**kw) == B.ERR_NULL, kw
    for kw in (dict(Q=FAKE + 2), dict(K=FAKE + 8), dict(Qo=FAKE + 4), dict(wq=FAKE + 2), dict(wk=FAKE + 8)):
        assert call(**kw) == B.ERR_ALIGN, kw
    for kw, want in BAD_ROPES:
        assert call(r=rope(B, **kw)) == getattr(B, want), kw


def test_norm_rope_backward_refusals(B):
    L = B.lib()
    need = B.patch_qk_norm_rope_backward_workspace_size(4, 8, 2, 128)
    assert need > 0

    def call(gQo=FAKE, ldgqo=1024, gKo=FAKE, ldgko=256, Q=FAKE, ldq=1024, Hq=8, K=FAKE, ldk=256, Hkv=2, M=4, D=128, wq=FAKE, wk=FAKE, r=rope(B),
             pos=FAKE, gQ=FAKE, ldgq=1024, gK=FAKE, ldgk=256, gwq=FAKE, gwk=FAKE, ws=FAKE, wsb=need):
        return L.patch_qk_norm_rope_backward(gQo, ldgqo, gKo, ldgko, Q, ldq, Hq, K, ldk, Hkv, M, D, wq, wk, 1e-6, r, pos, gQ, ldgq, gK, ldgk,
                                             gwq, gwk, ws, wsb, None, None)
    for kw in (dict(M=-1), dict(D=4), dict(Hq=-1), dict(ldq=1016), dict(ldgqo=1020), dict(ldgk=128)):
        assert call(**kw) == B.ERR_SHAPE, kw
    for kw in (dict(gQo=None), dict(gK=None), dict(Q=None), dict(K=None), dict(gwq=None), dict(gwk=None), dict(ws=None), dict(pos=None)):
        assert call(**kw) == B.ERR_NULL, kw
    for kw in (dict(Q=FAKE + 2), dict(gKo=FAKE + 8), dict(ws=FAKE + 16), dict(wq=FAKE + 2)):
        assert call(**kw) == B.ERR_ALIGN, kw
    assert call(wsb=need - 1) == B.ERR_SIZE
    for kw, want in BAD_ROPES:
        assert call(r=rope(B, **kw)) == getattr(B, want), kw
    n = ctypes.c_size_t(0)
    assert L.patch_qk_norm_rope_backward_workspace_size(4, 8, 2, 12, ctypes.byref(n)) == B.ERR_SHAPE
    assert L.patch_qk_norm_rope_backward_workspace_size(4, 8, 2, 128, None) == B.ERR_NULL


def test_append_refusals(B):
    L = B.lib()

    def call(c=cache(B), K=FAKE, ldk=256, V=FAKE, ldv=256, slots=FAKE, M=4, wk=None, r=rope(B), pos=FAKE, Q=FAKE, ldq=1024, Hq=8, wq=None, Qo=FAKE, ldqo=1024):
        return L.patch_kv_append(c, K, ldk, V, ldv, slots, M, wk, 1e-6, r, pos, Q, ldq, Hq, wq, Qo, ldqo, None, None)
    assert call(M=0, K=None, V=None, slots=None) == B.OK
    assert call(c=None) == B.ERR_NULL
    for kw, want in BAD_CACHES:
        assert call(c=cache(B, **kw)) == getattr(B, want), kw
    for kw, want in BAD_ROPES:
        assert call(r=rope(B, **kw)) == getattr(B, want), kw
    for kw in (dict(K=None), dict(V=None), dict(slots=None), dict(pos=None), dict(Q=None), dict(Qo=None)):
        assert call(**kw) == B.ERR_NULL, kw
    for kw in (dict(M=-1), dict(ldk=128), dict(ldv=252), dict(ldq=0), dict(Hq=-2)):
        assert call(**kw) == B.ERR_SHAPE, kw
    for kw in (dict(K=FAKE + 2), dict(V=FAKE + 8), dict(Q=FAKE + 2), dict(wk=FAKE + 2)):
        assert call(**kw) == B.ERR_ALIGN, kw


def test_attention_refusals(B):
    L = B.lib()
    c = cache(B)
    need = B.patch_prefix_attention_workspace_size(c, 3, 1, 8)
    assert need > 0

    def call(c=c, Q=FAKE, ldq=1024, n=3, T=1, Hq=8, pp=FAKE, P=100, table=FAKE, ld=4, lens=FAKE, scale=0.1, O=FAKE, ldo=1024, ws=FAKE, wsb=need):
        return L.patch_prefix_attention(c, Q, ldq, n, T, Hq, pp, P, table, ld, lens, scale, O, ldo, None, ws, wsb, None, None)
    assert call(n=0, Q=None, O=None, lens=None) == B.OK
    assert call(c=None) == B.ERR_NULL
    for kw, want in BAD_CACHES:
        assert call(c=cache(B, **kw)) == getattr(B, want), kw
    for kw in (dict(n=-1), dict(n=2049), dict(T=0), dict(Hq=7), dict(Hq=0), dict(P=-1), dict(P=1 << 31), dict(ld=-1), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(ldq=1016), dict(ldo=1028), dict(n=2048, T=1 << 20)):
        assert call(**kw) == B.ERR_SHAPE, kw
    assert call(c=cache(B, D=96)) == B.ERR_SHAPE
    for kw in (dict(Q=None), dict(O=None), dict(lens=None), dict(pp=None), dict(table=None), dict(ws=None)):
        assert call(**kw) == B.ERR_NULL, kw
    for kw in (dict(Q=FAKE + 2), dict(O=FAKE + 8), dict(ws=FAKE + 16)):
        assert call(**kw) == B.ERR_ALIGN, kw
    assert call(wsb=need - 1) == B.ERR_SIZE
    assert L.patch_prefix_attention_workspace_size(c, 3, 1, 8, None) == B.ERR_NULL
    with pytest.raises(B.PatchError):
        B.patch_prefix_attention_workspace_size(c, 3, 1, 9)


def test_tensors_are_checked_before_the_library_is_called(B):
    """The module that takes tensors apart: wrong types, shapes, layouts and devices are refused (a null function would be called last)."""
    torch = pytest.importorskip("torch")
    from paper_2509_23410_b200 import _marshal as m
    x = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    c = cache(B)
    at = ctypes.addressof(c)
    for bad in (x, x.float(), x[:, :, ::2], x[0], 5, "x", x.transpose(0, 1)):
        with pytest.raises(AssertionError):
            m.kv_append(0, at, bad, bad, None, None, 1e-6, None, None, None, None, None, None, 0)
        with pytest.raises(AssertionError):
            m.qk_norm_rope(0, bad, None, None, None, 1e-6, None, None, bad, None, None, 0)
        with pytest.raises(AssertionError):
            m.qk_norm_rope_backward(0, bad, None, None, None, None, None, 1e-6, None, None, bad, None, None, None, None, None, 0)
        with pytest.raises(AssertionError):
            m.prefix_attention(0, at, bad, None, 0, bad, bad, None, bad, None, None, None, 0)
    with pytest.raises(AssertionError):
        m.qk_norm_rope(0, None, None, None, None, 1e-6, None, None, None, None, None, 0)
    for f in (m.kv_append, m.qk_norm_rope, m.qk_norm_rope_backward, m.prefix_attention):
        with pytest.raises(TypeError):
            f(0)


def test_attention_scale_bound(B):
    """scale log2(e) has to be an fp32 number: twice that would be an infinity in every exponent."""
    L, c = B.lib(), cache(B)
    need = B.patch_prefix_attention_workspace_size(c, 3, 1, 8)
    call = lambda scale: L.patch_prefix_attention(c, FAKE, 1024, 3, 1, 8, FAKE, 100, FAKE, 4, FAKE, scale, FAKE, 1024, None, FAKE, need - 1, None, None)  # noqa: E731
    assert call(2.5e38) == B.ERR_SHAPE and call(1.9e38) == B.ERR_SIZE


def test_attention_counts_tiles_in_32_bits(B):
    """Refused before a device is touched, and only where the count would not fit."""
    L, c = B.lib(), cache(B, Hkv=8, page_stride=8 * 16 * 128)
    need = B.patch_prefix_attention_workspace_size(c, 2048, 1, 8)
    call = lambda n, P, ld: L.patch_prefix_attention(c, FAKE, 1024, n, 1, 8, FAKE, P, FAKE, ld, FAKE, 0.1, FAKE, 1024, None, FAKE, need, FAKE, None)  # noqa: E731
    wide = 8 * 1024 * 1024 // 16                              # pages of 16 keys: 8 million keys
    assert call(2048, 0, wide) == B.ERR_SHAPE and call(2048, 1 << 30, 4) == B.ERR_SHAPE and call(1, 100, 0x7FFFFFFF) == B.ERR_SHAPE
    import torch
    if not torch.cuda.is_available():                         # these are let through: the missing device is what is reported
        for args in ((2048, 0, wide - 600), (2047, 1 << 23, wide - 4200), (1, 0x7FFFFF00, 4)):
            assert call(*args) in (B.ERR_CUDA, B.ERR_ARCH), args
    assert call(1, 0x7FFFFF01, 4) == B.ERR_SHAPE
