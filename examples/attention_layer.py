"""The attention half of a decoder layer around the packed linear layers: serving a batch behind a shared prompt, and a training
step through the norms and the rotation.

    python examples/attention_layer.py                       # on a B200; prints what it checked and the time of a decode step

``Layer`` holds a stacked q/k/v projection and the o projection as packed tile-hybrid weights (dense and 2:4 tiles), weights of the
query and key norms, and a paged cache.  ``prompt`` writes the shared prompt to the cache once; ``step`` is one decode step of the
batch: q/k/v projection -> norms, rotation and append in one launch -> attention -> o projection.  ``QKNormRope`` is the training
form of the same norms and rotation as an autograd function.
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_23410_b200 import binding as B  # noqa: E402

BF = torch.bfloat16


def rope_table(positions: int, rotary_dim: int, base: float = 10000.0) -> torch.Tensor:
    freq = base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / rotary_dim)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * freq[None, :]
    return torch.cat((angle.cos(), angle.sin()), 1).float().cuda()


class QKNormRope(torch.autograd.Function):
    """(Q, K, wq, wk) -> normed and rotated (Q, K), with the gradient kernel behind it; a weight may be None (rotation alone)."""

    @staticmethod
    def forward(ctx, Q, K, wq, wk, rope, positions, eps):
        ctx.save_for_backward(Q if wq is not None else None, K if wk is not None else None, wq, wk, positions)
        ctx.rope, ctx.eps = rope, eps
        return B.patch_qk_norm_rope(Q, K, rope, positions, wq=wq, wk=wk, eps=eps)

    @staticmethod
    @torch.autograd.function.once_differentiable          # the gradient kernel is not differentiated in turn
    def backward(ctx, gQ, gK):
        Q, K, wq, wk, positions = ctx.saved_tensors
        gQ, gK, *gw = B.patch_qk_norm_rope_backward(gQ.contiguous(), gK.contiguous(), ctx.rope, positions, Q=Q, K=K, wq=wq, wk=wk, eps=ctx.eps)
        return gQ, gK, *(g if g is None else g.to(BF) for g in gw), None, None, None


class Layer:
    """Attention of one decoder layer for a batch of `batch` sequences that share a prompt."""

    def __init__(self, hidden: int, Hq: int, Hkv: int, D: int, batch: int, max_prompt: int, max_own: int, page: int = 16,
                 sparse: float = 0.5, seed: int = 0):
        self.Hq, self.Hkv, self.D, self.batch, self.page, self.hidden = Hq, Hkv, D, batch, page, hidden
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.linear = []
        for n, k in (((Hq + 2 * Hkv) * D, hidden), (hidden, Hq * D)):
            w = (torch.randn(n, k, generator=g, device="cuda") * 0.02).to(BF)
            flags = (rng.random((n // 128, k // 128)) < sparse).astype(np.uint8)
            packed, layout = B.patch_pack(w, flags)
            self.linear.append((layout, packed))
        self.ws = torch.zeros(max(B.patch_gemm_workspace_size(l, m) for l, _ in self.linear for m in (64, 65, max_prompt)), dtype=torch.uint8, device="cuda")
        self.wq, self.wk = ((1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(BF) for _ in range(2))
        self.rope = B.patch_rope(rope_table(max_prompt + max_own, D))
        own_pages = -(-max_own // page)
        self.prefix_pages = torch.arange(-(-max_prompt // page), dtype=torch.int32, device="cuda")
        first = self.prefix_pages.numel()
        self.table = (first + torch.randperm(batch * own_pages, generator=torch.Generator().manual_seed(seed)).view(batch, own_pages)).int().cuda()
        pages = first + batch * own_pages
        self.k, self.v = (torch.zeros(pages, Hkv, page, D, dtype=BF, device="cuda") for _ in range(2))
        self.cache = B.patch_kv_cache(self.k, self.v)
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.prefix_len = 0
        self.attn_ws = torch.empty(B.patch_prefix_attention_workspace_size(self.cache, batch, 1, Hq), dtype=torch.uint8, device="cuda")
        self.qkv, self.q = torch.empty(batch, (Hq + 2 * Hkv) * D, dtype=BF, device="cuda"), torch.empty(batch, Hq, D, dtype=BF, device="cuda")
        self.o, self.y = torch.empty_like(self.q), torch.empty(batch, hidden, dtype=BF, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def split(self, qkv):
        """Columns of the stacked projection as heads; nothing is copied."""
        Hq, Hkv, D = self.Hq, self.Hkv, self.D
        return (qkv[:, : Hq * D].unflatten(1, (Hq, D)), qkv[:, Hq * D : (Hq + Hkv) * D].unflatten(1, (Hkv, D)),
                qkv[:, (Hq + Hkv) * D :].unflatten(1, (Hkv, D)))

    def prompt(self, x):
        """Keys and values of the shared prompt's hidden states [P, hidden] into the prefix's pages."""
        P = x.shape[0]
        layout, packed = self.linear[0]
        qkv = B.patch_gemm(x, layout, packed, workspace=self.ws, status=self.status)
        _, k, v = self.split(qkv)
        at = torch.arange(P, device="cuda")
        slots = self.prefix_pages[at // self.page].long() * self.page + at % self.page
        B.patch_kv_append(self.cache, k, v, slots, rope=self.rope, positions=at.int(), wk=self.wk, status=self.status)
        self.prefix_len = P
        return qkv

    def place(self):
        """Slot and position of every sequence's next token."""
        n = self.lens.long()
        slots = self.table.gather(1, (n // self.page)[:, None]).squeeze(1).long() * self.page + n % self.page
        return slots, (self.prefix_len + self.lens).int()

    def step(self, x, slots, positions):
        """One decode step: hidden states [batch, hidden] of one new token per sequence -> the layer's attention output."""
        layout, packed = self.linear[0]
        B.patch_gemm(x, layout, packed, Y=self.qkv, workspace=self.ws, status=self.status, variant=B.VARIANT_AUTO | B.WEIGHTS_STATIC)
        q, k, v = self.split(self.qkv)
        B.patch_kv_append(self.cache, k, v, slots, rope=self.rope, positions=positions, wk=self.wk, Q=q, wq=self.wq, Q_out=self.q, status=self.status)
        self.lens += 1
        B.patch_prefix_attention(self.cache, self.q, self.prefix_pages, self.prefix_len, self.table, self.lens, O=self.o, workspace=self.attn_ws,
                                 status=self.status)
        layout, packed = self.linear[1]
        return B.patch_gemm(self.o.view(self.batch, -1), layout, packed, Y=self.y, workspace=self.ws, status=self.status,
                            variant=B.VARIANT_AUTO | B.WEIGHTS_STATIC)


def plain_attention(layer: Layer, prompt_qkv, own_qkv):
    """The same attention output of the newest token in plain 64-bit torch, from the projections alone."""
    def norm_turn(x, w, pos):
        x = x.double()
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.double()
        t = layer.rope.table[pos.long()].double()
        h = layer.D // 2
        c, s = t[:, None, :h], t[:, None, h:]
        return torch.cat((x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s), -1)
    P, n, G = layer.prefix_len, len(own_qkv), layer.Hq // layer.Hkv
    _, kp, vp = layer.split(prompt_qkv)
    kp = norm_turn(kp, layer.wk, torch.arange(P, device="cuda")).to(BF).double()
    out = []
    for b in range(layer.batch):
        rows = torch.stack([x[b] for x in own_qkv])
        q, k, v = layer.split(rows)
        pos = P + torch.arange(n, device="cuda")
        k = torch.cat((kp, norm_turn(k, layer.wk, pos).to(BF).double())).transpose(0, 1)
        v = torch.cat((vp.double(), v.double())).transpose(0, 1)
        q = norm_turn(q[-1:], layer.wq, pos[-1:]).to(BF).double().view(layer.Hkv, G, layer.D)
        p = torch.softmax(q @ k.transpose(1, 2) * layer.D ** -0.5, -1)
        out.append((p @ v).reshape(layer.Hq, layer.D))
    return torch.stack(out)


def serve(layer: Layer, prompt_len: int, steps: int, seed: int = 1) -> float:
    """A prompt and `steps` decode steps; returns the last step's attention error against the plain form, relative."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    prompt_qkv = layer.prompt(torch.randn(prompt_len, layer.hidden, generator=g, device="cuda").to(BF))
    own = []
    for _ in range(steps):
        slots, positions = layer.place()
        layer.step(torch.randn(layer.batch, layer.hidden, generator=g, device="cuda").to(BF), slots, positions)
        own.append(layer.qkv.clone())
    torch.cuda.synchronize()
    assert int(layer.status.item()) == 0, B.strerror(int(layer.status.item()))
    want = plain_attention(layer, prompt_qkv, own)
    return float((layer.o.double() - want).norm() / want.norm())


def train_step(M: int = 64, Hq: int = 8, Hkv: int = 2, D: int = 128, lr: float = 0.05, steps: int = 5):
    """Fits the norms' weights to a target through the gradient kernel; returns the losses."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rope, pos = B.patch_rope(rope_table(M, D)), torch.arange(M, dtype=torch.int32, device="cuda")
    q, k = (torch.randn(M, h, D, generator=g, device="cuda").to(BF) for h in (Hq, Hkv))
    target_q, target_k = B.patch_qk_norm_rope(q, k, rope, pos, wq=torch.full((D,), 1.5, dtype=BF, device="cuda"), wk=torch.full((D,), 0.5, dtype=BF, device="cuda"))
    w = [torch.ones(D, device="cuda", requires_grad=True) for _ in range(2)]
    losses = []
    for _ in range(steps):
        yq, yk = QKNormRope.apply(q, k, w[0].to(BF), w[1].to(BF), rope, pos, 1e-6)
        loss = ((yq.float() - target_q.float()).square().mean() + (yk.float() - target_k.float()).square().mean()) * D
        losses.append(float(loss.detach()))
        for p, gr in zip(w, torch.autograd.grad(loss, w)):
            p.data -= lr * gr * 8
    return losses


def main():
    layer = Layer(hidden=4096, Hq=32, Hkv=32, D=128, batch=16, max_prompt=2048, max_own=256)
    err = serve(layer, prompt_len=2000, steps=3)
    print(f"decode step of 16 sequences behind 2000 shared keys: attention within {err:.2e} of the plain form")
    slots, positions = layer.place()
    x = torch.randn(16, 4096, device="cuda").to(BF)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, slots, positions)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(3):
        graph.replay()
    start.record()
    for _ in range(50):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    print(f"q/k/v projection -> append -> attention -> o projection: {start.elapsed_time(end) / 50 * 1e3:.1f} us a step")
    print("training the norms' weights, losses:", " ".join(f"{v:.3f}" for v in train_step()))


if __name__ == "__main__":
    main()
