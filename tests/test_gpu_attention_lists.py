"""Attention's backward with lists of kept sequences that are not in order: every kernel keeps the same ones, those above all before them."""
import pytest
import torch

from paper_2402_17227_b200 import binding as vb
from tests.test_gpu_attention import BF16, F32, packed, tensors

pytestmark = pytest.mark.gpu


def kept_of(lst, n):
    kept = []
    for x in lst:
        if 0 <= x < n and x > (kept[-1] if kept else -1):
            kept.append(x)
    return kept


SHORT = [[0, 6, 1, 2], [1, 3, 2, 3], [5, 99, -1, 6], [7, 7, 7, 7, 7, 7, 7, 7], [3, 2, 1, 0], [-4, 8, 2], [4, 1, 5, 1, 6, 5, 7, 0]]
LONG = [[0, 5, 3] + list(range(6, 190, 3)) + [100, 190], list(range(0, 64, 2)) + [3] + list(range(64, 200, 7)), list(range(199, -1, -1)),
        list(range(31)) + [60] + list(range(31, 62))]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lst", SHORT + LONG, ids=lambda x: f"{len(x)}.{x[0]}.{x[1]}")
@pytest.mark.parametrize("skip", [False, True])
@pytest.mark.parametrize("equal", [False, True])
def test_a_list_out_of_order_keeps_what_it_says(dtype, D, lst, skip, equal):
    n = 8 if lst in SHORT else 200
    lens = [40] * n if equal else [(37 * i * i) % 91 for i in range(n)]
    starts, total = packed(lens), sum(lens)
    q, k, v = tensors(total, 2, 1, D, dtype, "plain", 8)
    do = tensors(total, 2, 1, D, dtype, "plain", 9)[0]
    op = vb.Attention(total, n, 2, 1, D, dtype, causal=True)
    o, lse = op.fwd(q, k, v, starts)

    def grads(entries):
        # what an earlier call left in the workspace is of no use to anyone
        op.bwd(100 * do, q, k, v, o, lse, starts)
        assert op.device_status() == 0
        out = [torch.full_like(x, 7.0) for x in (q, k, v)]
        a = torch.tensor(entries + [0] * (n - len(entries)), dtype=torch.int32, device="cuda")
        op.bwd(do, q, k, v, o, lse, starts, dq=out[0], dk=out[1], dv=out[2], alive_in=a,
               alive_cnt_in=torch.tensor([len(entries)], dtype=torch.int32, device="cuda"), skip_dropped_rows=skip)
        return out, op.device_status()

    kept = kept_of(lst, n)
    want, status = grads(kept)
    assert status == 0
    got, status = grads(lst)
    assert status == -1
    rows = torch.zeros(total, dtype=torch.bool, device="cuda")
    for i in kept:
        rows[int(starts[i]):int(starts[i + 1])] = True
    for a, b in zip(want, got):
        assert torch.equal(a, b)
        assert (b[~rows] == (7.0 if skip else 0.0)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_lists(dtype):
    """More entries than are gone through one by one: in order, and with one that is not."""
    n = 900
    lens = [(37 * i * i) % 23 for i in range(n)]
    starts, total = packed(lens), sum(lens)
    q, k, v = tensors(total, 2, 1, 64, dtype, "plain", 8)
    do = tensors(total, 2, 1, 64, dtype, "plain", 9)[0]
    op = vb.Attention(total, n, 2, 1, 64, dtype, causal=True)
    o, lse = op.fwd(q, k, v, starts)
    full = op.bwd(do, q, k, v, o, lse, starts)

    def grads(entries):
        out = [torch.full_like(x, 7.0) for x in (q, k, v)]
        a = torch.tensor(entries + [0] * (n - len(entries)), dtype=torch.int32, device="cuda")
        op.bwd(do, q, k, v, o, lse, starts, dq=out[0], dk=out[1], dv=out[2], alive_in=a,
               alive_cnt_in=torch.tensor([len(entries)], dtype=torch.int32, device="cuda"))
        return out, op.device_status()

    order = [i for i in range(n) if i % 7 != 3]
    for lst, status in (order, 0), (order[:600] + [order[5]] + order[600:], -1), (order[:300] + [880] + order[300:], -1):
        got, st = grads(lst)
        assert st == status
        rows = torch.zeros(total, dtype=torch.bool, device="cuda")
        for i in kept_of(lst, n):
            rows[int(starts[i]):int(starts[i + 1])] = True
        for a, b in zip(full, got):
            assert torch.equal(a[rows], b[rows]) and (b[~rows] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_more_sequences_than_tokens(dtype):
    """Entries behind the last tile are looked at too."""
    n, total = 200, 40
    starts = torch.tensor([min(i, total) for i in range(n + 1)], dtype=torch.int32, device="cuda")
    q, k, v = tensors(total, 2, 1, 64, dtype, "plain", 8)
    op = vb.Attention(total, n, 2, 1, 64, dtype, causal=True)
    o, lse = op.fwd(q, k, v, starts)
    assert op.device_status() == 0
    for lst, status in (list(range(n)), 0), (list(range(n - 1)) + [3], -1):
        got = op.bwd(q, q, k, v, o, lse, starts, alive_in=torch.tensor(lst, dtype=torch.int32, device="cuda"),
                     alive_cnt_in=torch.tensor([n], dtype=torch.int32, device="cuda"))
        assert op.device_status() == status
        # one key each: dV is dO of both heads, P = 1 to 2^-20, both sides rounded once
        a, b = q[:, :1].double(), q[:, 1:].double()
        assert ((got[2].double() - a - b).abs() <= 0.51 * torch.finfo(dtype).eps * (a + b).abs() + 2.0 ** -20 * (a.abs() + b.abs())).all()
    starts[n - 1] = 41
    op.fwd(q, k, v, starts)
    assert op.device_status() == -1
