"""One training step of mask logits on packed sequences: a decoder block whose weights pass through soft masks learns from the
dense block's most likely next tokens.

    python examples/learn_masks.py                           # on a B200; prints the time of a step and of its parts

``Block`` holds frozen weights of the stacked q/k/v projection and the o projection, an output matrix, and the mask logits that
learn.  ``Block.logits`` is soft masks -> projection -> norms and rotation -> attention within the packed sequences -> o projection
-> output matrix; with ``dense=True`` the same with the weights as they are, which is the teacher.  ``step`` takes the teacher's
list, both losses and the gradients of the mask logits.  Rows behind the last sequence are padding: attention leaves them alone, so
its results and gradients are made of zeros here, and their tokens are -1.
"""
from __future__ import annotations

import os
import sys

import torch
from torch.autograd.function import once_differentiable

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paper_2509_23410_b200 import binding as B  # noqa: E402

BF = torch.bfloat16


class SoftMask(torch.autograd.Function):
    """(W, P_tile, P24) -> the softly masked weight; gradients of the two kinds of logits (of the loss alone: the regularisers' share
    goes into the same call by its two coefficients)."""

    @staticmethod
    def forward(ctx, W, P_tile, P24, tau, kappa, seed, flags):
        ctx.save_for_backward(W, P_tile, P24)
        ctx.how = tau, kappa, seed, flags
        return B.patch_soft_mask(W, P_tile, P24, tau, kappa, seed=seed, flags=flags)[0]

    @staticmethod
    @once_differentiable
    def backward(ctx, gWt):
        tau, kappa, seed, flags = ctx.how
        gP_tile, gP24 = B.patch_soft_mask_backward(*ctx.saved_tensors, tau, kappa, gWt.contiguous(), 0.0, 0.0, seed=seed, flags=flags)
        return None, gP_tile, gP24, None, None, None, None


class QKNormRope(torch.autograd.Function):
    """(Q, K, wq, wk) -> normed and rotated (Q, K); the norms' weights are frozen here."""

    @staticmethod
    def forward(ctx, Q, K, wq, wk, rope, positions):
        ctx.save_for_backward(Q, K, wq, wk, positions)
        ctx.rope = rope
        return B.patch_qk_norm_rope(Q, K, rope, positions, wq=wq, wk=wk)

    @staticmethod
    @once_differentiable
    def backward(ctx, gQ, gK):
        Q, K, wq, wk, positions = ctx.saved_tensors
        gQ, gK, *_ = B.patch_qk_norm_rope_backward(gQ.contiguous(), gK.contiguous(), ctx.rope, positions, Q=Q, K=K, wq=wq, wk=wk)
        return gQ, gK, None, None, None, None


class SequenceAttention(torch.autograd.Function):
    """(Q, K, V, starts) -> O; padding rows are 0 in the result and in the gradients."""

    @staticmethod
    def forward(ctx, Q, K, V, starts):
        lse = torch.empty(Q.shape[:2], device=Q.device)
        O = B.patch_sequence_attention(Q, K, V, starts, O=torch.zeros(Q.shape, dtype=BF, device=Q.device), lse=lse)
        ctx.save_for_backward(Q, K, V, O, lse, starts)
        return O

    @staticmethod
    @once_differentiable
    def backward(ctx, gO):
        Q, K, V, O, lse, starts = ctx.saved_tensors
        g = [torch.zeros(t.shape, dtype=BF, device=t.device) for t in (Q, K, V)]
        B.patch_sequence_attention_backward(gO.contiguous(), Q, K, V, O, lse, starts, gQ=g[0], gK=g[1], gV=g[2])
        return *g, None


class TokenLogprobs(torch.autograd.Function):
    """(Z, tokens) -> (log probabilities, entropies) of the rows."""

    @staticmethod
    def forward(ctx, Z, tokens, temperature):
        logp, entropy, lse, _, _ = B.patch_token_logprobs(Z, tokens, temperature=temperature, entropy=True, lse=True)
        ctx.save_for_backward(Z, tokens, lse, entropy)
        ctx.temperature = temperature
        return logp, entropy

    @staticmethod
    @once_differentiable
    def backward(ctx, glogp, gentropy):
        Z, tokens, lse, entropy = ctx.saved_tensors
        return B.patch_token_logprobs_backward(Z, tokens, lse, glogp.contiguous(), entropy, gentropy.contiguous(), ctx.temperature), None, None


class DistillLoss(torch.autograd.Function):
    """(Z, ids, logp) -> cross entropy of every row with the teacher's list."""

    @staticmethod
    def forward(ctx, Z, ids, logp, temperature, rest):
        stats = torch.empty(Z.shape[0], 2, device=Z.device)
        ctx.save_for_backward(Z, ids, logp, stats)
        ctx.how = temperature, rest
        return B.patch_distill_loss(Z, ids, logp, temperature, rest, stats=stats)

    @staticmethod
    @once_differentiable
    def backward(ctx, gloss):
        return B.patch_distill_loss_backward(*ctx.saved_tensors, gloss.contiguous(), *ctx.how), None, None, None, None


class Block:
    """Attention of a decoder layer with an output matrix over V columns (V need be no multiple of anything)."""

    def __init__(self, hidden: int, Hq: int, Hkv: int, D: int, V: int, positions: int, seed: int = 0):
        self.Hq, self.Hkv, self.D, self.V = Hq, Hkv, D, V
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.W = [(rand(n, k) * k ** -0.5).to(BF) for n, k in (((Hq + 2 * Hkv) * D, hidden), (hidden, Hq * D))]
        self.masks = []
        for w in self.W:
            n, k = w.shape
            self.masks.append((rand(n // 128, k // 128).requires_grad_(), rand(6, n * k // 4).requires_grad_()))
        self.out = (rand(-(-V // 8) * 8, hidden) * hidden ** -0.5).to(BF)         # logits' rows start at multiples of 16 bytes
        self.wq, self.wk = ((1 + 0.1 * rand(D)).to(BF) for _ in range(2))
        freq = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
        angle = torch.arange(positions, dtype=torch.float64)[:, None] * freq
        self.rope = B.patch_rope(torch.cat((angle.cos(), angle.sin()), 1).float().cuda())

    def weights(self, tau: float, kappa: float, seed: int, flags: int):
        return [SoftMask.apply(w, pt, p24, tau, kappa, seed + i, flags) for i, (w, (pt, p24)) in enumerate(zip(self.W, self.masks))]

    def logits(self, x, starts, positions, weights):
        Hq, Hkv, D = self.Hq, self.Hkv, self.D
        qkv = (x @ weights[0].T).unflatten(1, (-1, D))
        q, k, v = qkv.split((Hq, Hkv, Hkv), 1)                     # columns of the projection; nothing is copied
        q, k = QKNormRope.apply(q, k, self.wq, self.wk, self.rope, positions)
        o = SequenceAttention.apply(q, k, v, starts)
        y = x + o.flatten(1) @ weights[1].T
        return (y @ self.out.T)[:, : self.V]


def positions_of(starts, M: int):
    """Position of each row within its sequence (padding: from 0 again)."""
    row = torch.arange(M, device=starts.device)
    own = torch.searchsorted(starts.long(), row, right=True) - 1
    return torch.where(own < 0, row, row - starts.long()[own.clamp(min=0)]).int()


def step(block: Block, x, starts, tokens, k: int = 32, temperature: float = 1.5, share: float = 0.5, rest: bool = True, tau: float = 2.0,
         kappa: float = 25.0, seed: int = 0, flags: int = 0):
    """share of the distillation and 1 - share of the tokens' own loss, mean over the rows that count -> (loss, gradients of the mask
    logits, the teacher's list)."""
    positions = positions_of(starts, x.shape[0])
    with torch.no_grad():
        teacher = block.logits(x, starts, positions, block.W)
        *_, ids, logp = B.patch_token_logprobs(teacher, k=k, temperature=temperature)
        counts = tokens >= 0
        ids.masked_fill_(~counts[:, None], -1)
    z = block.logits(x, starts, positions, block.weights(tau, kappa, seed, flags))
    distilled = DistillLoss.apply(z, ids, logp, temperature, rest)
    own, _ = TokenLogprobs.apply(z, tokens, 1.0)
    loss = (share * distilled - (1 - share) * own).masked_fill(~counts, 0.0).sum() / counts.sum()
    return loss.detach(), torch.autograd.grad(loss, [p for pair in block.masks for p in pair]), (ids, logp)


def batch(M: int, lens, hidden: int, V: int, seed: int = 1):
    """Hidden states, sequence starts and next tokens of packed sequences of these lengths, padded to M rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, hidden, generator=g, device="cuda").to(BF)
    starts = torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda")
    tokens[starts[1:].long() - 1] = -1                             # a sequence's last row has no next token
    tokens[sum(lens):] = -1
    return x, starts, tokens


def main():
    hidden, Hq, Hkv, D, V, M, lens = 4096, 32, 32, 128, 32000, 4096, (1700, 1100, 640, 400, 200)
    block = Block(hidden, Hq, Hkv, D, V, M)
    x, starts, tokens = batch(M, lens, hidden, V)
    for _ in range(3):
        loss, grads, _ = step(block, x, starts, tokens)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    start.record()
    for i in range(10):
        step(block, x, starts, tokens, seed=2 * i)
    end.record()
    torch.cuda.synchronize()
    print(f"{sum(lens)} tokens of {len(lens)} sequences, {V} columns: loss {float(loss):.4f}, {start.elapsed_time(end) / 10:.2f} ms a step, gradient norms "
          + " ".join(f"{float(g.norm()):.2e}" for g in grads))


if __name__ == "__main__":
    main()
