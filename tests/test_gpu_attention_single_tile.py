"""Attention's backward where a tile of rows has a single tile of keys, heads wider than 64: its two halves of delta are exchanged while
those of the next rows may be on their way."""
import pytest
import torch

from paper_2402_17227_b200 import binding as vb
from tests.attn_ref import check, reference
from tests.test_gpu_attention import BF16, packed, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens", [[128] * 40, [1 + (37 * i) % 128 for i in range(300)], [100, 300, 64, 129, 128, 500, 1] * 20])
def test_the_same_bits_over_and_over(causal, lens):
    starts, total = packed(lens), sum(lens)
    q, k, v = tensors(total, 4, 2, 128, BF16, "fused", 1)
    do = tensors(total, 4, 2, 128, BF16, "plain", 2)[0]
    op = vb.Attention(total, len(lens), 4, 2, 128, BF16, causal=causal)
    o, lse = op.fwd(q, k, v, starts)
    first = op.bwd(do, q, k, v, o, lse, starts)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(first, op.bwd(do, q, k, v, o, lse, starts)))
    few = 5                                           # sequences that the reference looks at
    T = sum(lens[:few])
    st = packed(lens[:few])
    ref = reference(q[:T], k[:T], v[:T], st, causal, 128 ** -0.5, do[:T])
    for name, got in zip(("dq", "dk", "dv"), op.bwd(do, q, k, v, o, lse, starts)):
        check(got[:T], ref[name], what=name)
    assert op.device_status() == 0
