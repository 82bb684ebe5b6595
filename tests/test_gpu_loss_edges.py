"""Calls from packed sequences to a loss that the documentation allows at its edges: what lies beside a sequence, masked columns under large factors, temperatures and
logits of any size.  References and tolerances are those of test_gpu_logits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF = torch.bfloat16

from test_gpu_logits import B  # noqa: E402, F401


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 40, 130, 300])
def test_rows_beside_a_sequence_leave_its_bits_alone(B, D, n):  # noqa: F811
    """The rows behind a sequence share tiles with its last ones; whatever they hold, results and gradients are the same bits.  Here their scores with the
    sequence's keys rise steeply, so that their maxima are raised again and again."""
    Hq, Hkv, M = 4, 2, 512
    g = torch.Generator(device="cuda").manual_seed(n)
    q, k, v, go = (torch.randn(M, h, D, generator=g, device="cuda").to(BF) for h in (Hq, Hkv, Hkv, Hq))
    k[:n] += torch.linspace(0, 2, n, device="cuda")[:, None, None].to(BF)
    got = []
    for other in (0.0, 1.0, 30.0, -30.0, math.nan):
        q[n:] = other
        for starts in ([0, n], [0, n, M]):
            where = torch.tensor(starts, dtype=torch.int32, device="cuda")
            lse = torch.zeros(M, Hq, device="cuda")
            o = B.patch_sequence_attention(q, k, v, where, O=torch.zeros_like(q), lse=lse)
            grads = B.patch_sequence_attention_backward(go, q, k, v, o, lse, where)
            got.append([x[:n].clone() for x in (o, lse, *grads)])
    for other in got[1:]:
        # (the gradients of keys are summed in as many parts as the number of sequences suggests: equal numbers of them are compared)
        assert all(torch.equal(a, b) for a, b in zip(got[0][:3], other[:3]))
    assert all(torch.equal(a, b) for first in (0, 1) for i in range(first, len(got), 2) for a, b in zip(got[first], got[i]))
