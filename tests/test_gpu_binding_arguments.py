"""Arguments that are no numbers are refused by the calls between the linear layers before anything is launched."""
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


@pytest.mark.parametrize("eps", ["1e-6", None, [1e-6]])
def test_eps(B, eps):
    x = torch.randn(5, 6, 64, device="cuda").to(BF)
    w, out = torch.ones(64, dtype=BF, device="cuda"), torch.full((5, 6, 64), 3.0, dtype=BF, device="cuda")
    k, v = (torch.full((2, 6, 16, 64), 3.0, dtype=BF, device="cuda") for _ in range(2))
    cache, slots = B.patch_kv_cache(k, v), torch.arange(5, device="cuda")
    gw = torch.full((64,), 3.0, device="cuda")
    with pytest.raises(TypeError):
        B.patch_qk_norm_rope(x, None, None, None, wq=w, eps=eps, Q_out=out)
    with pytest.raises(TypeError):
        B.patch_qk_norm_rope_backward(x, None, None, None, Q=x, wq=w, eps=eps, gQ=out, gwq=gw)
    with pytest.raises(TypeError):
        B.patch_kv_append(cache, x, x, slots, wk=w, eps=eps, Q=x, Q_out=out)
    torch.cuda.synchronize()
    assert all(bool((t == 3.0).all()) for t in (out, k, v, gw))


@pytest.mark.parametrize("kw", [dict(scale="0.1"), dict(scale=[0.1]), dict(prefix_len=1.5), dict(prefix_len=1 << 70)])
def test_scale_and_prefix_length(B, kw):
    k, v = (torch.zeros(4, 2, 16, 64, dtype=BF, device="cuda") for _ in range(2))
    cache, q = B.patch_kv_cache(k, v), torch.zeros(1, 2, 64, dtype=BF, device="cuda")
    o = torch.full((1, 2, 64), 3.0, dtype=BF, device="cuda")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    args = dict(prefix_pages=i32(0, 1), prefix_len=20, page_table=i32(2).view(1, 1), suffix_lens=i32(3), O=o) | kw
    with pytest.raises((TypeError, OverflowError)):
        B.patch_prefix_attention(cache, q, **args)
    torch.cuda.synchronize()
    assert bool((o == 3.0).all())
