"""The calls from packed sequences to a loss on streams of the caller's: memory that they allocate by themselves, several at once, and the whole chain
captured and replayed with other contents."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2509_23410_b200 import build, binding as b
    build.build()
    return b


def rand(seed, *shape, dtype=BF):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


class Chain:
    """Heads of two packed sequences and logits of as many rows; `shape` decides which kernels the logits take."""

    def __init__(self, seed, M, V, dtype):
        self.M = M
        self.q, self.k, self.v, self.go = (rand(seed + i, M, h, 64) for i, h in enumerate((4, 2, 2, 4)))
        self.z, self.t = rand(seed + 4, M, V, dtype=dtype), rand(seed + 5, M, V, dtype=dtype)
        self.starts = torch.tensor([0, M // 3, M], dtype=torch.int32, device="cuda")
        self.tokens = torch.arange(M, device="cuda") * 7 % V
        self.one = torch.ones(M, device="cuda")

    def all(self, B, stream=None):
        kw = dict(stream=stream)
        lse = torch.empty(self.M, 4, device="cuda") if stream is None else B._empty(stream, (self.M, 4), torch.float32, "cuda")
        stats = torch.empty(self.M, 2, device="cuda") if stream is None else B._empty(stream, (self.M, 2), torch.float32, "cuda")
        o = B.patch_sequence_attention(self.q, self.k, self.v, self.starts, lse=lse, **kw)
        grads = B.patch_sequence_attention_backward(self.go, self.q, self.k, self.v, o, lse, self.starts, **kw)
        logp, entropy, zl, ids, top = B.patch_token_logprobs(self.t, self.tokens, k=9, entropy=True, lse=True, **kw)
        gt = B.patch_token_logprobs_backward(self.t, self.tokens, zl, self.one, entropy, self.one, **kw)
        loss = B.patch_distill_loss(self.z, ids, top, rest=True, stats=stats, **kw)
        gz = B.patch_distill_loss_backward(self.z, ids, top, stats, rest=True, **kw)
        both = torch.empty_like(self.z) if stream is None else B._empty(stream, self.z.shape, self.z.dtype, "cuda")
        B.patch_distill_loss(self.z, ids, top, rest=True, loss=loss, gZ=both, **kw)
        return o, *grads, logp, entropy, zl, ids, top, gt, loss, gz, both


SHAPES = [(5, 1000, BF), (300, 32000, BF), (40, 128256, torch.float32), (600, 128256, BF)]        # the last: rows that stay in shared memory


@pytest.mark.parametrize("M,V,dtype", SHAPES)
def test_own_memory_and_two_streams_at_once(B, monkeypatch, M, V, dtype):
    chains = [Chain(10 * i, M, V, dtype) for i in (1, 2)]
    want = [c.all(B) for c in chains]
    torch.cuda.synchronize()
    real, seen = B._empty, []

    def empty(stream, *a):
        seen.append(stream)
        return real(stream, *a)
    monkeypatch.setattr(B, "_empty", empty)
    streams, got = [torch.cuda.Stream() for _ in chains], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for i, (c, s) in enumerate(zip(chains, streams)):
            seen.clear()
            got.append((i, c.all(B, stream=s)))
            assert len(seen) >= 15 and all(x is s for x in seen)
            torch.empty_like(c.z).fill_(float("nan"))              # the current stream's own memory, written meanwhile
    torch.cuda.synchronize()
    for i, r in got:
        assert all(torch.equal(a, b) for a, b in zip(r, want[i]))


@pytest.mark.parametrize("M,V,dtype", SHAPES[:3])
def test_captured_chain_follows_its_contents(B, M, V, dtype):
    c, other = Chain(1, M, V, dtype), Chain(50, M, V, dtype)
    other.starts = torch.tensor([1, M // 2, M - 1], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.all(B)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.all(B)
    for name in ("q", "k", "v", "go", "z", "t", "starts"):
        getattr(c, name).copy_(getattr(other, name))
    graph.replay()
    want = other.all(B)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        rows = slice(1, M - 1) if i < 4 else slice(None)           # rows outside the sequences are not written
        assert torch.equal(a[rows], b[rows]), i
