"""What small problems show in one launch, on the kernels of the others: decode kernel, block kernel, joining kernel, and the two or three
of them that one call launches.  Strided results and scales of one's own, captured launches that follow their lengths, other streams, lengths
and pages out of range.  Tolerances: those of ``Batch.check``."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_attention import BF, B, Batch  # noqa: E402,F401  (B is a fixture)

pytestmark = pytest.mark.gpu

# lens, T, Hq, Hkv, D, P, page, extra pages in the table (room for 160000 keys keeps the small kernel away)
PATHS = {
    "decode, own keys": ([100, 333, 64, 200], 2, 8, 2, 128, 0, 16, 10000),
    "decode, prefix and own keys": ([100, 333, 64, 200], 1, 8, 2, 64, 700, 32, 5000),
    "block for the prefix, decode": ([5, 40, 0, 130] * 9, 1, 8, 2, 128, 16001, 16, 10000),
    "block for both": ([400, 333, 90, 200], 40, 8, 2, 128, 300, 64, 2500),
    "block, a prompt": ([700, 600, 64, 520], 516, 2, 1, 64, 0, 16, 10000),
}


@pytest.fixture(params=PATHS)
def case(request):
    return PATHS[request.param]


def batch(B, case, seed, **kw):
    lens, T, Hq, Hkv, D, P, page, extra = case
    return Batch(B, list(lens), T, Hq, Hkv, D, P, page, seed=seed, extra=extra, **kw)


def test_result_pitch_and_scale(B, case):
    """A strided result leaves its gaps alone; the scale is the caller's; the workspace is the call's own."""
    x = batch(B, case, 3, q_scale=4.0, pitch=64)
    n, wide = x.q.shape[0], x.Hq * x.D
    buf = torch.full((n, wide + 64), 7.0, dtype=BF, device="cuda")
    o, l = buf[:, :wide].unflatten(1, (x.Hq, x.D)), torch.empty(n, x.Hq, device="cuda")
    B.patch_prefix_attention(x.cache, x.q, x.prefix_pages, x.P, x.table, x.len_dev, O=o, lse=l, scale=0.21)
    torch.cuda.synchronize()
    x.check(o, l, scale=0.21)
    assert bool((buf[:, wide:] == 7.0).all())


def test_captured_launches_follow_the_lengths(B, case):
    x = batch(B, case, 4)
    n = x.q.shape[0]
    o, l = torch.empty(n, x.Hq, x.D, dtype=BF, device="cuda"), torch.empty(n, x.Hq, device="cuda")
    ws = torch.empty(B.patch_prefix_attention_workspace_size(x.cache, len(x.lens), x.T, x.Hq), dtype=torch.uint8, device="cuda")
    call = lambda: B.patch_prefix_attention(x.cache, x.q, x.prefix_pages, x.P, x.table, x.len_dev, O=o, lse=l, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    own = list(x.lens)
    for lens in (own, [0] * len(own), [min(n, 1) if i % 3 else n for i, n in enumerate(own)], [n // 2 for n in own], [max(0, n - 1) for n in own], own):
        x.len_dev.copy_(torch.tensor(lens, dtype=torch.int32))
        x.lens = lens
        kept = x.ks
        x.ks = [k[:n] for k, n in zip(kept, lens)]
        ws.fill_(0xFF)
        g.replay()
        g.replay()                                             # and once more right behind it, on the same workspace
        torch.cuda.synchronize()
        x.check(o, l)
        x.ks = kept


def test_on_another_stream(B, case):
    x = batch(B, case, 5)
    want, _ = x.run(B)
    s = torch.cuda.Stream()
    o = torch.zeros_like(want)
    ws = torch.empty(B.patch_prefix_attention_workspace_size(x.cache, len(x.lens), x.T, x.Hq), dtype=torch.uint8, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    B.patch_prefix_attention(x.cache, x.q, x.prefix_pages, x.P, x.table, x.len_dev, O=o, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(o, want)


def test_lengths_and_pages_out_of_range(B, case):
    """Reported, and nothing is read out of bounds: a length is clamped, page 0 read for one that is not there.  The next call is right."""
    x = batch(B, case, 6)
    want, want_l = x.run(B)

    def call(status, **kw):
        o, l = torch.full_like(want, 7.0), torch.full_like(want_l, 7.0)
        a = dict(prefix=x.prefix_pages, table=x.table, lens=x.len_dev) | kw
        B.patch_prefix_attention(x.cache, x.q, a["prefix"], x.P, a["table"], a["lens"], O=o, lse=l, status=status)
        return o, l
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for bad, as_if in ((-3, 0), (-2 ** 31, 0)):
        status.zero_()
        lens = x.len_dev.clone()
        lens[1] = bad
        o, l = call(status, lens=lens)
        assert int(status.item()) == B.ERR_SIZE
        lens[1] = as_if
        o2, l2 = call(None, lens=lens)
        assert torch.equal(o, o2) and torch.equal(l, l2)
    room = x.table.shape[1] * x.page
    table = x.table.clone()
    table[1] = x.table[1, 0]                                   # every entry a page of the cache: the clamped length is a legal one
    for bad in (room + 1, 2 ** 31 - 1):
        status.zero_()
        lens = x.len_dev.clone()
        lens[1] = bad
        o, l = call(status, lens=lens, table=table)
        assert int(status.item()) == B.ERR_SIZE
        lens[1] = room
        status.zero_()
        o2, l2 = call(status, lens=lens, table=table)
        assert int(status.item()) == B.OK
        rows = torch.arange(x.q.shape[0], device="cuda") // x.T != 1       # NaN in sequence 1: its table repeats a page that may end in NaN
        assert torch.equal(o[rows], o2[rows]) and torch.equal(l[rows], l2[rows])
    for bad in (x.k.shape[0], -1, 2 ** 31 - 1, -2 ** 31):
        status.zero_()
        table = x.table.clone()
        table[1, 0] = bad
        call(status, table=table)
        assert int(status.item()) == B.ERR_FORMAT
        if x.P:
            status.zero_()
            prefix = x.prefix_pages.clone()
            prefix[len(prefix) // 2] = bad
            call(status, prefix=prefix)
            assert int(status.item()) == B.ERR_FORMAT
    status.zero_()
    o, l = call(status)
    assert int(status.item()) == B.OK and torch.equal(o, want) and torch.equal(l, want_l)
