"""Attention with starts that make no sense in places: the sequences there are left out, forward and backward, and the others' results
are theirs."""
import pytest
import torch

from paper_2402_17227_b200 import binding as vb
from tests.attn_ref import check, reference
from tests.test_gpu_attention import BF16, F32, packed, tensors

pytestmark = pytest.mark.gpu
TOTAL, HQ, HK = 200, 4, 2
# starts, and the sequences among them that can be followed: (place in the list, first token, end)
CASES = [([0, 60, -3, 60, 200], [(0, 0, 60), (3, 60, 200)]),
         ([0, 60, 500, 60, 200], [(0, 0, 60), (3, 60, 200)]),
         ([-3, 100, 150, 200], [(1, 100, 150), (2, 150, 200)]),
         ([0, 100, 150, 201], [(0, 0, 100), (1, 100, 150)]),
         ([0, 70, 70, -1, -1, 70, 71, 200], [(0, 0, 70), (5, 70, 71), (6, 71, 200)])]


def run(dtype, layout, D, case, kept):
    """kept: None for all, or the one of this number among those that can be followed alone."""
    bad, good = CASES[case]
    starts = torch.tensor(bad, dtype=torch.int32, device="cuda")
    N = len(bad) - 1
    sane = torch.tensor([good[0][1]] + [e for _, _, e in good], dtype=torch.int32)
    q, k, v = tensors(TOTAL, HQ, HK, D, dtype, layout, 1)
    do = tensors(TOTAL, HQ, HK, D, dtype, layout, 2)[0]
    op = vb.Attention(TOTAL, N, HQ, HK, D, dtype, causal=True)
    mark = 7.0
    fill = lambda seed: [t.fill_(mark) for t in tensors(TOTAL, HQ, HK, D, dtype, layout, seed)]
    ref = reference(q, k, v, sane, True, D ** -0.5, do, None if kept is None else [kept])
    inside = torch.zeros(TOTAL, dtype=torch.bool, device="cuda")
    inside[good[0][1]:good[-1][2]] = True
    o, lse = fill(3)[0], torch.full((HQ, TOTAL), mark, device="cuda")
    op.fwd(q, k, v, starts, o=o, lse=lse)
    assert op.device_status() == -1 and op.device_status() == 0
    check(o, ref["o"], inside, "o")
    check(lse.T, tuple(x.T for x in ref["lse"]), inside, "lse")
    assert (o[~inside] == mark).all() and (lse[:, ~inside] == mark).all()
    # what an earlier call left in the workspace is of no use to anyone
    far = tensors(TOTAL, HQ, HK, D, dtype, layout, 4)[0].mul_(100)
    op.bwd(far, q, k, v, far, lse.fill_(0), packed([TOTAL]))
    assert op.device_status() == 0
    kw = {}
    if kept is not None:
        kw = dict(alive_in=torch.tensor([good[kept][0]] + [0] * (N - 1), dtype=torch.int32, device="cuda"),
                  alive_cnt_in=torch.ones(1, dtype=torch.int32, device="cuda"))
    # as the formulas have o and lse, so that the backward's own error is what is measured
    o.copy_(ref["o"][0])
    outs = fill(5)
    op.bwd(do, q, k, v, o, ref["lse"][0].float(), starts, dq=outs[0], dk=outs[1], dv=outs[2], **kw)
    assert op.device_status() == -1 and op.device_status() == 0
    mine = inside if kept is None else torch.zeros_like(inside)
    if kept is not None:
        mine[good[kept][1]:good[kept][2]] = True
    for name, got in zip(("dq", "dk", "dv"), outs):
        check(got, ref[name], mine, name)
        assert (got[~inside] == mark).all(), name
        dropped = got[inside & ~mine]                 # set to zero, or left
        assert ((dropped == 0) | (dropped == mark)).all(), name


@pytest.mark.parametrize("dtype,layout", [(F32, "plain"), (F32, "odd"), (BF16, "plain"), (BF16, "odd")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_other_sequences_keep_their_results(dtype, layout, D, case):
    run(dtype, layout, D, case, None)


@pytest.mark.parametrize("dtype,layout", [(F32, "plain"), (F32, "odd"), (BF16, "plain"), (BF16, "odd")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("kept", [0, 1])
def test_a_kept_one_keeps_its_results(dtype, layout, D, case, kept):
    run(dtype, layout, D, case, kept)
