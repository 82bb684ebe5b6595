"""Attention of a batch behind a shared prefix over the paged cache on the GPU, against the definition in 64 bits.

Tolerances.  A probability is rounded to bf16 for its product with V (2^-8 of it at most) and the result once more (2^-8 of the
result); a score is a sum of D products accumulated in fp32, so it is off by at most D 2^-24 of the sum of its terms' sizes, which
enters a probability as twice that (numerator and sum); exponentials, sums and joins of parts add 2^-17 at most."""
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


class Batch:
    """A batch in a cache whose every slot that holds no key of it is NaN; pages in random order, tables padded with -1."""

    def __init__(self, B, lens, T, Hq, Hkv, D, P, page, seed=0, shared_buffer=False, pitch=0, q_scale=1.5, extra=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = len(lens)
        self.lens, self.T, self.P, self.page, self.D, self.Hq, self.Hkv = lens, T, P, page, D, Hq, Hkv
        used = -(-P // page)
        count = [-(-x // page) for x in lens]
        pool = used + sum(count) + 2
        if shared_buffer:
            both = torch.full((pool, 2, Hkv, page, D), float("nan"), dtype=BF, device="cuda")
            self.k, self.v = both[:, 0], both[:, 1]
        else:
            self.k, self.v = (torch.full((pool, Hkv, page, D), float("nan"), dtype=BF, device="cuda") for _ in range(2))
        order = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).tolist()
        fill = lambda m: torch.randn(m, Hkv, D, generator=g, device="cuda").to(BF)  # noqa: E731
        self.kp, self.vp = fill(P), fill(P)
        self.ks, self.vs = [fill(x) for x in lens], [fill(x) for x in lens]
        self.prefix_pages = torch.tensor(order[:used], dtype=torch.int32, device="cuda")
        self._put(order[:used], self.kp, self.vp)
        width = max(count + [1]) + extra
        table = torch.full((n, width), -1, dtype=torch.int32)
        at = used
        for b in range(n):
            mine = order[at : at + count[b]]
            at += count[b]
            table[b, : count[b]] = torch.tensor(mine, dtype=torch.int32)
            self._put(mine, self.ks[b], self.vs[b])
        self.table = table.cuda()
        self.len_dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.q = (torch.randn(n * T, Hq * D + pitch, generator=g, device="cuda") * q_scale).to(BF)[:, : Hq * D].unflatten(1, (Hq, D))
        self.cache = B.patch_kv_cache(self.k, self.v)

    def _put(self, pages, k, v):
        for i, p in enumerate(pages):
            rows = slice(i * self.page, min((i + 1) * self.page, k.shape[0]))
            m = rows.stop - rows.start
            self.k[p, :, :m] = k[rows].transpose(0, 1)
            self.v[p, :, :m] = v[rows].transpose(0, 1)

    def run(self, B, lse=True, **kw):
        o = torch.full((self.q.shape[0], self.Hq, self.D), 7.0, dtype=BF, device="cuda")
        l = torch.full((self.q.shape[0], self.Hq), 7.0, device="cuda") if lse else None
        ws = torch.full((B.patch_prefix_attention_workspace_size(self.cache, len(self.lens), self.T, self.Hq),), 0xFF, dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.patch_prefix_attention(self.cache, self.q, self.prefix_pages, self.P, self.table, self.len_dev, O=o, lse=l, workspace=ws,
                                 status=status, **kw)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        return o, l

    def check(self, o, l, scale=None):
        scale = self.D ** -0.5 if scale is None else scale
        G, T = self.Hq // self.Hkv, self.T
        for b in range(len(self.lens)):
            k = torch.cat((self.kp, self.ks[b])).double().transpose(0, 1)            # [Hkv, n, D]
            v = torch.cat((self.vp, self.vs[b])).double().transpose(0, 1)
            for t in range(T):
                n = self.P + max(0, self.lens[b] - (T - 1 - t))
                row = b * T + t
                if n == 0:
                    assert float(o[row].float().abs().max()) == 0.0
                    assert l is None or bool((l[row] == -float("inf")).all())
                    continue
                q = self.q[row].double().view(self.Hkv, G, self.D)
                s = q @ k[:, :n].transpose(1, 2) * scale
                ds = (q.abs() @ k[:, :n].abs().transpose(1, 2) * scale).amax(-1, keepdim=True) * self.D * 2.0 ** -24
                m = s.amax(-1, keepdim=True)
                p = (s - m).exp()
                den = p.sum(-1, keepdim=True)
                ref, size = p @ v[:, :n] / den, p @ v[:, :n].abs() / den
                tol = ref.abs() * 2.0 ** -8 * 1.01 + size * (2.0 ** -8 + 2 * ds + 2.0 ** -17) + 1e-30
                err = (o[row].double().view(self.Hkv, G, self.D) - ref).abs()
                assert bool((err <= tol).all()), (b, t, float((err / tol).nan_to_num(1e9).max()))
                if l is not None:
                    want = (m + den.log()).view(-1)
                    assert bool(((l[row].double() - want).abs() <= ds.view(-1) + 2.0 ** -17 + want.abs() * 2.0 ** -22).all())


CASES = [  # lens, T, Hq, Hkv, D, P, page
    ([1], 1, 1, 1, 128, 0, 16),
    ([0], 1, 4, 4, 128, 1, 16),
    ([0, 0, 3], 1, 4, 2, 64, 0, 16),                       # rows that see nothing
    ([0, 1, 2, 3, 4, 5], 4, 8, 2, 128, 0, 32),             # drafted tokens, some of which see nothing
    ([17, 64, 65, 1, 128, 127], 1, 32, 32, 128, 128, 16),
    ([63, 200, 5], 1, 16, 2, 128, 63, 64),
    ([63, 200, 5], 1, 16, 2, 64, 64, 128),
    ([300, 2, 31, 33], 3, 12, 4, 64, 65, 256),
    ([9, 700, 40], 5, 8, 1, 128, 257, 32),                 # 40 rows of one key head and sequence
    ([1000], 7, 40, 40, 128, 777, 16),
    ([5] * 33, 1, 8, 2, 128, 2000, 16),                    # 132 rows against the prefix
    ([129] * 40, 1, 8, 1, 64, 900, 64),
    ([1 + 37 * i % 301 for i in range(64)], 1, 4, 1, 128, 4000, 16),
    ([2, 900, 1, 1, 450] * 20, 1, 5, 5, 128, 130, 128),
    ([65] * 3, 1, 64, 64, 64, 5000, 32),
    ([40] * 2, 16, 64, 8, 128, 300, 16),                   # 128 rows of one key head and sequence
    ([260] * 2, 33, 8, 1, 128, 129, 16),                   # 264 rows of one, a third block of them partly filled
    ([3], 1, 8, 8, 128, 20000, 16),                        # one sequence, a long prefix: an item over many SMs
    ([0] * 300, 1, 4, 4, 64, 70, 16),                      # no own keys at all
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("layout", ["plain", "strided"])
def test_against_the_definition(B, case, layout):
    lens, T, Hq, Hkv, D, P, page = CASES[case]
    kw = dict(shared_buffer=True, pitch=2 * Hkv * D, extra=3) if layout == "strided" else {}
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case, **kw)
    o, l = x.run(B)
    x.check(o, l)
    o2, _ = x.run(B, lse=False)
    assert torch.equal(o, o2), "equal calls give equal bits"


@pytest.mark.parametrize("case", range(len(CASES)))
def test_behind_wide_tables(B, case):
    """The kernels are chosen by the width of the page table: the same batches with room for 160000 keys a sequence, which takes none
    of them into the single launch of small problems."""
    lens, T, Hq, Hkv, D, P, page = CASES[case]
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case, extra=160000 // page)
    o, l = x.run(B)
    x.check(o, l)
    o2, _ = x.run(B, lse=False)
    assert torch.equal(o, o2), "equal calls give equal bits"


LONG = [  # prefixes whose rows and keys are the block kernel's
    ([5] * 33, 1, 8, 2, 128, 20000, 16),
    ([1 + 37 * i % 301 for i in range(64)], 1, 4, 1, 128, 17001, 16),
    ([129] * 40, 1, 8, 1, 64, 16000, 64),
    ([300, 2, 31, 33] * 4, 3, 12, 4, 64, 9000, 256),
    ([0] * 300, 1, 4, 4, 64, 13000, 16),
]


@pytest.mark.parametrize("case", range(len(LONG)))
def test_long_prefixes(B, case):
    lens, T, Hq, Hkv, D, P, page = LONG[case]
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case)
    o, l = x.run(B)
    x.check(o, l)
    o2, _ = x.run(B, lse=False)
    assert torch.equal(o, o2), "equal calls give equal bits"


SMALL = [  # lens, T, Hq, Hkv, D, P, page: from one CTA to sixteen an item, items beyond the CTAs that run at once
    ([8000], 1, 8, 1, 128, 0, 16),
    ([500], 1, 16, 2, 128, 4000, 64),
    ([16000, 3, 0, 5000], 4, 8, 2, 64, 0, 256),
    ([1] * 37, 1, 8, 8, 128, 1, 16),
    ([0, 100] * 37, 1, 32, 8, 128, 100, 32),
    ([64 * i + i % 3 for i in range(9)], 2, 8, 1, 64, 64, 128),
    ([65] * 4, 3, 15, 3, 128, 127, 64),
    ([40, 700], 7, 16, 2, 128, 300, 16),                   # 56 rows: four blocks of them
    ([90], 64, 3, 3, 64, 5, 32),
]


@pytest.mark.parametrize("case", range(len(SMALL)))
@pytest.mark.parametrize("layout", ["plain", "strided"])
def test_small_problems(B, case, layout):
    lens, T, Hq, Hkv, D, P, page = SMALL[case]
    kw = dict(shared_buffer=True, pitch=2 * Hkv * D, extra=3) if layout == "strided" else {}
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case, **kw)
    o, l = x.run(B)
    x.check(o, l)
    o2, _ = x.run(B, lse=False)
    assert torch.equal(o, o2), "equal calls give equal bits"


PROMPTS = [  # many tokens a sequence: row blocks that see different numbers of tiles
    ([513], 513, 4, 1, 64, 0, 32),
    ([600, 65, 0, 10], 530, 4, 2, 128, 70, 16),            # more tokens than keys: the first ones see nothing
    ([1500, 640, 639], 640, 3, 1, 128, 200, 64),           # blocks of 128 rows that begin within a token
    ([257] * 5, 65, 16, 2, 128, 0, 128),
    ([600, 1, 128, 127], 520, 3, 3, 64, 129, 16),
]


@pytest.mark.parametrize("case", range(len(PROMPTS)))
def test_prompts(B, case):
    lens, T, Hq, Hkv, D, P, page = PROMPTS[case]
    x = Batch(B, lens, T, Hq, Hkv, D, P, page, seed=case)
    o, l = x.run(B)
    x.check(o, l)
    o2, _ = x.run(B, lse=False)
    assert torch.equal(o, o2), "equal calls give equal bits"


def test_result_pitch_scale_and_peaked_scores(B):
    """A strided result leaves its gaps alone; a scale of one's own; scores far apart (the maximum moves and parts differ by
    hundreds of powers of two)."""
    x = Batch(B, [100, 333, 64], 1, 8, 2, 128, 500, 16, seed=3, q_scale=30.0)
    wide = torch.full((3, 8 * 128 + 64), 7.0, dtype=BF, device="cuda")
    l = torch.empty(3, 8, device="cuda")
    B.patch_prefix_attention(x.cache, x.q, x.prefix_pages, x.P, x.table, x.len_dev, O=wide[:, :1024].unflatten(1, (8, 128)), lse=l, scale=0.37)
    torch.cuda.synchronize()
    x.check(wide[:, :1024].unflatten(1, (8, 128)), l, scale=0.37)
    assert bool((wide[:, 1024:] == 7.0).all())


def test_captured_launch_follows_the_lengths(B):
    x = Batch(B, [100, 333, 64, 200], 1, 8, 2, 128, 200, 16, seed=4)
    o, l = torch.empty(4, 8, 128, dtype=BF, device="cuda"), torch.empty(4, 8, device="cuda")
    ws = torch.empty(B.patch_prefix_attention_workspace_size(x.cache, 4, 1, 8), dtype=torch.uint8, device="cuda")
    call = lambda: B.patch_prefix_attention(x.cache, x.q, x.prefix_pages, x.P, x.table, x.len_dev, O=o, lse=l, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for lens in ([100, 333, 64, 200], [1, 300, 0, 7], [99, 1, 64, 200]):
        x.len_dev.copy_(torch.tensor(lens, dtype=torch.int32))
        x.lens = lens
        g.replay()
        torch.cuda.synchronize()
        x.check(o, l)


def test_on_another_stream(B):
    x = Batch(B, [100, 333], 1, 8, 2, 128, 200, 16, seed=5)
    want, _ = x.run(B)
    s = torch.cuda.Stream()
    o = torch.zeros_like(want)
    s.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(B.patch_prefix_attention_workspace_size(x.cache, 2, 1, 8), dtype=torch.uint8, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    B.patch_prefix_attention(x.cache, x.q, x.prefix_pages, x.P, x.table, x.len_dev, O=o, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(o, want)


def test_lengths_and_pages_outside_their_range_are_reported(B):
    """Bounds are checked before anything is read: a length is clamped, a page replaced by page 0."""
    x = Batch(B, [20, 30], 1, 4, 2, 64, 40, 16, seed=6)
    for lens, want in (([-3, 30], B.ERR_SIZE), ([20, 10 ** 6], B.ERR_SIZE)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        B.patch_prefix_attention(x.cache, x.q, x.prefix_pages, x.P, x.table, n, status=status)
        assert int(status.item()) == want
    bad = x.table.clone()
    bad[1, 0] = x.k.shape[0]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.patch_prefix_attention(x.cache, x.q, x.prefix_pages, x.P, bad, x.len_dev, status=status)
    assert int(status.item()) == B.ERR_FORMAT
    bad = x.prefix_pages.clone()
    bad[0] = -7
    status.zero_()
    B.patch_prefix_attention(x.cache, x.q, bad, x.P, x.table, x.len_dev, status=status)
    assert int(status.item()) == B.ERR_FORMAT


def test_empty_batch(B):
    x = Batch(B, [20], 1, 4, 2, 64, 40, 16, seed=7)
    q = torch.empty(0, 4, 64, dtype=BF, device="cuda")
    o = B.patch_prefix_attention(x.cache, q, x.prefix_pages, 40, x.table[:0], x.len_dev[:0])
    assert o.shape == (0, 4, 64)
