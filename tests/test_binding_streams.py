"""Memory that the calls between the linear layers allocate by themselves comes from the allocator's share of the stream they run on.
On the CPU: a recording stand-in for torch's allocator and for the module that launches.  On the GPU: calls on several streams at once, each
with a workspace of the call's own."""
import types

import pytest

torch = pytest.importorskip("torch")


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle

    def __eq__(self, other):
        return isinstance(other, Stream) and other.cuda_stream == self.cuda_stream


class Recorder:
    """What torch.empty and torch.cuda.stream do, as far as the binding uses them: a tensor knows the stream it was allocated for."""

    def __init__(self):
        self.now, self.made = "current", []
        rec = self

        class On:
            def __init__(self, s):
                self.s = s

            def __enter__(self):
                self.before, rec.now = rec.now, self.s

            def __exit__(self, *a):
                rec.now = self.before
        self.cuda = types.SimpleNamespace(stream=On, Stream=Stream, ExternalStream=lambda handle, device: Stream(handle))
        self.uint8, self.float32 = torch.uint8, torch.float32

    def empty(self, shape, dtype=None, device=None):
        self.made.append(self.now)
        return types.SimpleNamespace(shape=shape)


@pytest.mark.parametrize("stream", [None, Stream(77), types.SimpleNamespace(cuda_stream=77)])
def test_own_memory_belongs_to_the_calls_stream(monkeypatch, stream):
    from paper_2509_23410_b200 import build
    build.build()
    from paper_2509_23410_b200 import binding as B
    rec, launched = Recorder(), []

    def launch(*a):
        launched.append(a[-1])
        return B.OK
    monkeypatch.setattr(B, "_torch", rec)
    monkeypatch.setattr(B, "_bf16", torch.bfloat16)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 5)
    monkeypatch.setattr(B, "_marshal", types.SimpleNamespace(qk_norm_rope=launch, qk_norm_rope_backward=launch, kv_append=launch, prefix_attention=launch))
    x = types.SimpleNamespace(shape=(4, 2, 128), device="cuda", get_device=lambda: 0)
    w = object()
    cache = B.KVCache(1 << 20, 1 << 20, 10, 2 * 16 * 128, 16, 2, 128, 0)
    cache.at = 0
    table = types.SimpleNamespace(shape=(4, 3))
    B.patch_qk_norm_rope(x, x, None, None, stream=stream)                                # both results
    B.patch_qk_norm_rope_backward(x, x, None, None, Q=x, K=x, wq=w, wk=w, stream=stream)  # two gradients each, a workspace
    B.patch_kv_append(cache, x, x, None, Q=x, stream=stream)                             # the queries
    B.patch_prefix_attention(cache, x, None, 0, table, None, stream=stream)              # the result, a workspace
    assert launched == [5 if stream is None else 77] * 4
    assert rec.made == ["current" if stream is None else Stream(77)] * 10


@pytest.mark.gpu
def test_streams_with_workspaces_of_their_own():
    """Two streams run attention and gradients at the same time while the current stream allocates and writes as much memory."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2509_23410_b200 import build, binding as B
    build.build()
    from test_gpu_attention import Batch
    x = [Batch(B, [700, 64, 333] * 6, 1, 8, 2, 128, 3000 + 700 * i, 16, seed=i, extra=10000) for i in range(2)]
    q = [torch.randn(3000, 16, 128, device="cuda").bfloat16() for _ in range(2)]
    w = torch.ones(128, device="cuda").bfloat16()
    attend = lambda i, **kw: B.patch_prefix_attention(x[i].cache, x[i].q, x[i].prefix_pages, x[i].P, x[i].table, x[i].len_dev, **kw)  # noqa: E731
    back = lambda i, **kw: B.patch_qk_norm_rope_backward(q[i], None, None, None, Q=q[1 - i], wq=w, **kw)  # noqa: E731
    want = [(attend(i), *back(i)[::2]) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(20):
        for i, s in enumerate(streams):
            got.append((i, attend(i, stream=s), *back(i, stream=s)[::2]))
        for n in (B.patch_prefix_attention_workspace_size(x[0].cache, 18, 1, 8), B.patch_qk_norm_rope_backward_workspace_size(3000, 16, 0, 128)):
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0xFF)
    torch.cuda.synchronize()
    for i, *r in got:
        assert all(torch.equal(a, b) for a, b in zip(r, want[i]))


@pytest.mark.gpu
def test_every_call_allocates_for_its_stream(monkeypatch):
    """The calls on weights and masks as well: each of them asks for its memory with the stream that it runs on, and is right there."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2509_23410_b200 import build, binding as B
    build.build()
    real, seen = B._empty, []

    def empty(stream, *a):
        seen.append(stream)
        return real(stream, *a)
    monkeypatch.setattr(B, "_empty", empty)
    N = K = 256
    g = torch.Generator(device="cuda").manual_seed(1)
    W, X, Gw = (torch.randn(r, K, generator=g, device="cuda").bfloat16() for r in (N, 5, N))
    P_tile, P24 = torch.randn(2, 2, generator=g, device="cuda"), torch.randn(6, N * K // 4, generator=g, device="cuda")
    flags = [0, 1, 1, 0]
    workspace = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    flags_dev = torch.tensor(flags, dtype=torch.uint8, device="cuda")

    def calls(stream):
        packed, layout = B.patch_pack(W, flags, stream=stream)
        kw = dict(workspace=workspace, stream=stream)
        hard, patterns = B.patch_hard_mask(P_tile, P24, N, K, stream=stream)
        return [packed, B.patch_unpack(layout, packed, stream=stream), B.patch_gemm(X, layout, packed, **kw),
                B.patch_gemm_gated(X, layout, packed, **kw), hard, patterns, B.patch_pack_patterns(W, flags, patterns, stream=stream)[0],
                *B.patch_soft_mask(W, P_tile, P24, 1.0, 1.0, stream=stream),
                *B.patch_soft_mask_backward(W, P_tile, P24, 1.0, 1.0, Gw, 0.1, 0.1, stream=stream),
                B.patch_unpack(layout, B.patch_pack_dev(W, flags_dev, stream=stream), stream=stream)]
    want = calls(None)
    torch.cuda.synchronize()
    count = len(seen)
    assert seen == [None] * count and count >= len(want)
    s = torch.cuda.Stream()
    for stream in (s, types.SimpleNamespace(cuda_stream=s.cuda_stream)):
        seen.clear()
        s.wait_stream(torch.cuda.current_stream())
        got = calls(stream)
        torch.cuda.synchronize()
        assert len(seen) == count and all(t is stream for t in seen)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
