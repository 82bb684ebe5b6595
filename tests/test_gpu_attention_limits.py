"""The attention-side operators at their limits: offsets beyond 32 bits, the largest batch, waits that run out (in the
fault-injection build; nothing faults or hangs: the waits are bounded and the launches complete)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
from test_gpu_attention import BF, B, Batch  # noqa: E402,F401  (B is a fixture)

pytestmark = pytest.mark.gpu
INJECT_MAGIC = 0x7E57


def test_offsets_beyond_32_bits(B):
    """Pages two gibibytes apart: byte and element offsets of the later pages pass 2^32 and 2^31."""
    Hkv, page, D, pages = 2, 16, 128, 6
    stride = (1 << 30) - 8                               # elements
    buf = torch.zeros((pages - 1) * stride + 2 * Hkv * page * D, dtype=BF, device="cuda")
    k = buf.as_strided((pages, Hkv, page, D), (stride, page * D, D, 1))
    v = buf.as_strided((pages, Hkv, page, D), (stride, page * D, D, 1), Hkv * page * D)
    assert (pages - 1) * stride > 1 << 32
    cache = B.patch_kv_cache(k, v)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(pages * page, 3 * Hkv, D, generator=g, device="cuda").to(BF)
    slots = torch.arange(pages * page, device="cuda")
    q = B.patch_kv_append(cache, x[:, Hkv : 2 * Hkv], x[:, 2 * Hkv :], slots, Q=x[:, :Hkv])
    for p in range(pages):
        assert torch.equal(k[p], x[p * page : (p + 1) * page, Hkv : 2 * Hkv].transpose(0, 1))
        assert torch.equal(v[p], x[p * page : (p + 1) * page, 2 * Hkv :].transpose(0, 1))
    assert torch.equal(q, x[:, :Hkv])
    # attention: prefix in the last two pages (again and again), own keys in the first ones; tables as wide as needed (one launch for all)
    # and wider (decode kernel; block kernel for the long prefix)
    for n, width, times in ((1, 2, 1), (33, 2, 1), (1, 10000, 1), (33, 10000, 1), (33, 2, 1400)):
        prefix = torch.tensor([pages - 1, pages - 2] * times, dtype=torch.int32, device="cuda")
        P = 2 * page * times - 2
        table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        table[:, :2] = torch.arange(2, dtype=torch.int32, device="cuda")
        lens = torch.full((n,), 20, dtype=torch.int32, device="cuda")
        qq = x[:n, :Hkv].contiguous()
        o = B.patch_prefix_attention(cache, qq, prefix, P, table, lens)
        order = torch.cat((torch.cat((slots[(pages - 1) * page :], slots[(pages - 2) * page : (pages - 1) * page])).repeat(times)[:P], slots[:20]))
        kk, vv = x[order, Hkv : 2 * Hkv].double().transpose(0, 1), x[order, 2 * Hkv :].double().transpose(0, 1)
        p = torch.softmax(torch.einsum("bhd,hnd->bhn", qq.double(), kk) * D ** -0.5, -1)
        ref, size = torch.einsum("bhn,hnd->bhd", p, vv), torch.einsum("bhn,hnd->bhd", p, vv.abs())
        assert bool(((o.double() - ref).abs() <= ref.abs() * 2.0 ** -8 * 1.01 + size * (2.0 ** -8 + 2.0 ** -12)).all())


def test_largest_batch(B):
    lens = [1 + 7 * i % 40 for i in range(2048)]
    x = Batch(B, lens, 1, 2, 1, 64, 100, 16, seed=9)
    o, l = x.run(B)
    x.lens = lens
    # a sample of the sequences: the check walks them one by one
    for b in list(range(0, 2048, 97)) + [2047]:
        k = torch.cat((x.kp, x.ks[b])).double().transpose(0, 1)
        v = torch.cat((x.vp, x.vs[b])).double().transpose(0, 1)
        q = x.q[b].double().view(1, 2, 64)
        p = torch.softmax(q @ k.transpose(1, 2) / 8.0, -1)
        ref, size = (p @ v)[0], (p @ v.abs())[0]
        assert bool(((o[b].double() - ref).abs() <= ref.abs() * 2.0 ** -8 * 1.01 + size * (2.0 ** -8 + 2.0 ** -12)).all()), b


@pytest.mark.parametrize("shape", [(1, 4, 4, 0), (1, 4, 4, 300), (40, 4, 1, 26000)])
@pytest.mark.parametrize("extra", [0, 10000])
def test_a_wait_that_runs_out_is_reported_and_survivable(B, shape, extra):
    """A CTA of the call's first kernel (the kernel of small problems; with wide tables the decode kernel; the block kernel for the 160
    rows of the last shape) waits for bytes that never come: it gives up, the launch completes with PATCH_ERR_TIMEOUT, the next
    call is right."""
    from paper_2509_23410_b200 import build
    n, Hq, Hkv, P = shape
    fi = B.load(build.build(fault_injection=True))
    x = Batch(B, [70] * n, 1, Hq, Hkv, 128, P, 16, seed=5, extra=extra)
    want, _ = x.run(B)
    ws = torch.full((B.patch_prefix_attention_workspace_size(x.cache, n, 1, Hq),), 0xFF, dtype=torch.uint8, device="cuda")
    o = torch.zeros_like(want)
    vp = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731

    def call(status):
        rc = fi.patch_prefix_attention(x.cache, vp(x.q), Hq * 128, n, 1, Hq, vp(x.prefix_pages) if P else None, P, vp(x.table), x.table.shape[1],
                                       vp(x.len_dev), 128 ** -0.5, vp(o), Hq * 128, None, vp(ws), ws.numel(), vp(status),
                                       ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == B.OK
        torch.cuda.synchronize()
        return int(status.item())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert call(status) == B.OK and torch.equal(o, want)
    status.fill_(INJECT_MAGIC)
    assert call(status) == B.ERR_TIMEOUT
    status.zero_()
    assert call(status) == B.OK and torch.equal(o, want)


@pytest.mark.parametrize("n", [615, 616, 1231, 1232, 2048])
@pytest.mark.parametrize("P", [0, 100, 4100])
def test_batches_around_the_limits_of_shared_memory(B, n, P):
    """Up to 615 sequences the decode kernel keeps their lengths, up to 1231 two of its CTAs fit an SM (heads of 128); alone, and beside the
    block kernel, which has the longer prefix."""
    lens = [(1 + 7 * i % 150) * (i % 11 != 3) for i in range(n)]
    x = Batch(B, lens, 1, 2, 1, 128, P, 16, seed=n)
    o, l = x.run(B)
    if P == 0:
        assert float(o[3].float().abs().max()) == 0.0 and bool((l[3] == -float("inf")).all())
    # a sample of the sequences: the check walks them one by one
    rows = [b for b in range(0, n, 41) if P or lens[b]] + [n - 1]
    x.lens, x.ks, x.vs = [lens[b] for b in rows], [x.ks[b] for b in rows], [x.vs[b] for b in rows]
    x.q = x.q[rows]
    x.check(o[rows], l[rows])
