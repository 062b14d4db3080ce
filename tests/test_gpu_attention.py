"""Attention over packed sequences against its formulas in 64 bits: lengths, heads, widths, strides, kept sequences, refusals."""
import math

import pytest
import torch

from tests.attn_ref import check, reference
from paper_2402_17227_b200 import binding as vb

pytestmark = pytest.mark.gpu


def packed(lens, device="cuda"):
    st = [0]
    for n in lens:
        st.append(st[-1] + n)
    return torch.tensor(st, dtype=torch.int32, device=device)


def tensors(total, Hq, Hk, D, dtype, layout, seed=0):
    """q, k, v of `total` tokens: separate, in one buffer, head by head, or with strides that TMA cannot address."""
    g = torch.Generator("cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)
    if layout == "fused":
        x = randn(total, Hq + 2 * Hk, D)
        return x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    if layout == "heads":
        return tuple(randn(h, total, D).transpose(0, 1) for h in (Hq, Hk, Hk))
    if layout == "odd":
        return tuple(randn(total, h, D + 3)[:, :, 1:D + 1] for h in (Hq, Hk, Hk))
    return randn(total, Hq, D), randn(total, Hk, D), randn(total, Hk, D)


def run(lens, Hq, Hk, D, dtype, causal, layout="plain", alive=None, behind=0, skip=False, seed=0):
    starts = packed(lens)
    T = int(starts[-1])
    total = T + behind
    q, k, v = tensors(total, Hq, Hk, D, dtype, layout, seed)
    do = tensors(total, Hq, Hk, D, dtype, layout, seed + 1)[0]
    for x in (q, k, v, do):
        x[T:] = float("nan")                 # nothing behind the last sequence is read
    scale = 1.0 / math.sqrt(D)
    op = vb.Attention(max(1, total), len(lens), Hq, Hk, D, dtype, causal=causal)
    mark = 7.0
    outs = [t.fill_(mark) for t in tensors(total, Hq, Hk, D, dtype, layout, seed + 2)]
    o = tensors(total, Hq, Hk, D, dtype, layout, seed + 3)[0].fill_(mark)
    lse = torch.full((Hq, total), mark, device="cuda")
    op.fwd(q, k, v, starts, o=o, lse=lse)
    ref = reference(q[:T], k[:T], v[:T], starts, causal, scale, do[:T], alive)
    check(o[:T], ref["o"], what="o")
    check(lse[:, :T], ref["lse"], what="lse")
    kw = {}
    if alive is not None:
        a = torch.full((len(lens),), -5, dtype=torch.int32, device="cuda")
        a[:len(alive)] = torch.tensor(alive, dtype=torch.int32)
        kw = dict(alive_in=a, alive_cnt_in=torch.tensor([len(alive)], dtype=torch.int32, device="cuda"), skip_dropped_rows=skip)
    # the backward on the formula's o and lse, so that its own error is what is measured
    ob, lb = ref["o"][0].to(dtype), ref["lse"][0].float()
    o_in = tensors(total, Hq, Hk, D, dtype, layout, seed + 4)[0].fill_(float("nan"))
    o_in[:T] = ob
    l_in = torch.full((Hq, total), float("nan"), device="cuda")
    l_in[:, :T] = lb
    op.bwd(do, q, k, v, o_in, l_in, starts, dq=outs[0], dk=outs[1], dv=outs[2], **kw)
    assert op.device_status() == 0
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    if skip:
        for n in range(len(lens)):
            if n not in alive:
                rows[int(starts[n]):int(starts[n + 1])] = False
    for name, got in zip(("dq", "dk", "dv"), outs):
        check(got[:T], ref[name], rows, name)
        assert (got[:T][~rows] == mark).all() and (got[T:] == mark).all(), name
    assert (o[T:] == mark).all() and (lse[:, T:] == mark).all()
    op.close()


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [8, 64, 72, 128])
def test_lengths_and_widths(dtype, causal, D):
    run([1, 63, 0, 128, 129, 2, 200], 2, 1, D, dtype, causal, behind=5)


@pytest.mark.parametrize("layout", ["fused", "heads", "odd"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(layout, dtype):
    run([100, 257, 31], 4, 2, 64, dtype, True, layout, behind=3)


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (8, 8), (8, 1), (6, 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_heads(Hq, Hk, causal):
    run([197, 40, 300], Hq, Hk, 128, BF16, causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("alive", [[], [0], [1, 3], [0, 1, 2, 3, 4]])
@pytest.mark.parametrize("skip", [False, True])
def test_kept_sequences(dtype, alive, skip):
    run([70, 130, 0, 257, 5], 4, 2, 64, dtype, True, "fused", alive=alive, skip=skip, behind=9)


@pytest.mark.parametrize("lens", [[0], [0, 0, 3, 0], [1], [1] * 70, [513], [1024, 1]])
def test_few_and_many_sequences(lens):
    run(lens, 2, 2, 64, BF16, False)
    run(lens, 2, 1, 128, BF16, True)


def test_long_sequence_keeps_its_precision():
    run([3000], 1, 1, 128, BF16, True)
    run([2500], 1, 1, 64, BF16, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_scores(dtype):
    """Rows whose maximum keeps rising tile by tile, and scores far from 0: the running maximum has to follow."""
    T, D = 600, 64
    g = torch.Generator("cuda").manual_seed(3)
    q = torch.randn(T, 1, D, generator=g, device="cuda")
    k = torch.randn(T, 1, D, generator=g, device="cuda")
    k = k + q.mean(0) * 0 + (torch.arange(T, device="cuda")[:, None, None] / 64.0) * torch.sign(q[:1])
    q = q.abs() * torch.sign(q[:1]) * 1.5
    v = torch.randn(T, 1, D, generator=g, device="cuda")
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    starts = packed([T])
    op = vb.Attention(T, 1, 1, 1, D, dtype)
    o, lse = op.fwd(q, k, v, starts)
    ref = reference(q, k, v, starts, False, 1.0 / 8.0)
    check(o, ref["o"], what="o")
    check(lse, ref["lse"], what="lse")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_sequence_keeps_its_nan_to_itself(dtype, bad):
    lens = [100, 60, 90]
    starts = packed(lens)
    q, k, v = tensors(250, 2, 2, 64, dtype, "fused", 5)
    do = tensors(250, 2, 2, 64, dtype, "plain", 6)[0]
    op = vb.Attention(250, 3, 2, 2, 64, dtype, causal=False)
    clean = [x.clone() for x in op.fwd(q, k, v, starts)]
    grads = [x.clone() for x in op.bwd(do, q, k, v, *clean, starts)]
    for x in (q, k, v, do):
        x[100:160] = bad
    o, lse = op.fwd(q, k, v, starts)
    d = op.bwd(do, q, k, v, o, lse, starts)
    rest = torch.cat([torch.arange(0, 100), torch.arange(160, 250)]).cuda()
    assert torch.equal(o[rest], clean[0][rest]) and torch.equal(lse[:, rest], clean[1][:, rest])
    for a, b in zip(d, grads):
        assert torch.equal(a[rest], b[rest])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_same_bits_twice_and_captured(dtype):
    lens = [300, 17, 129, 256]
    starts = packed(lens)
    T = sum(lens)
    q, k, v = tensors(T, 4, 2, 64, dtype, "fused", 8)
    do = tensors(T, 4, 2, 64, dtype, "plain", 9)[0]
    op = vb.Attention(T, 4, 4, 2, 64, dtype, causal=True)
    o, lse = op.fwd(q, k, v, starts)
    d = op.bwd(do, q, k, v, o, lse, starts)
    first = [x.clone() for x in (o, lse, *d)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op.fwd(q, k, v, starts, o=o, lse=lse)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.fwd(q, k, v, starts, o=o, lse=lse)
        op.bwd(do, q, k, v, o, lse, starts, dq=d[0], dk=d[1], dv=d[2])
    for x in (o, lse, *d):
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (o, lse, *d)))
    # the graph follows the data: other sequences in the same buffers
    starts.copy_(packed([200, 200, 200, T - 600]))
    graph.replay()
    torch.cuda.synchronize()
    ref = reference(q, k, v, starts, True, 0.125, do)
    check(o, ref["o"], what="o")
    assert op.device_status() == 0
    del graph


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_against_differences(dtype):
    """dL of a small step along a random direction, by the gradient and by the 64-bit formula."""
    lens, Hq, Hk, D = [37, 150], 2, 1, 64
    starts = packed(lens)
    T = sum(lens)
    q, k, v = tensors(T, Hq, Hk, D, dtype, "plain", 11)
    do = tensors(T, Hq, Hk, D, dtype, "plain", 12)[0]
    op = vb.Attention(T, 2, Hq, Hk, D, dtype, causal=True)
    o, lse = op.fwd(q, k, v, starts)
    grads = op.bwd(do, q, k, v, o, lse, starts)
    g = torch.Generator("cuda").manual_seed(13)
    loss = lambda a, b, c: float((reference(a, b, c, starts, True, 0.125)["o"][0] * do.double()).sum())
    h = 1e-4
    for i in range(3):
        x = [q.double(), k.double(), v.double()]
        d = torch.randn(x[i].shape, generator=g, device="cuda", dtype=torch.float64)
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + h * d, x[i] - h * d
        # `reference` takes its roundings from the type only for bounds: the values are those of the 64-bit inputs
        diff = (loss(*up) - loss(*down)) / (2 * h)
        got = float((grads[i].double() * d).sum())
        # per element off by at most the reference's bound; along d that is at most its dot product with |d|
        ref = reference(q, k, v, starts, True, 0.125, do)[("dq", "dk", "dv")[i]]
        slack = float((ref[1] * d.abs()).sum()) * 2 + 1e-5 * abs(diff)
        assert abs(got - diff) <= slack, (i, got, diff, slack)


def test_bad_starts_are_reported_and_not_followed():
    q, k, v = tensors(200, 2, 2, 64, BF16, "plain", 14)
    op = vb.Attention(200, 3, 2, 2, 64, BF16)
    o = torch.full_like(q, 7.0)
    for bad in ([0, 100, 50, 200], [-3, 100, 150, 200], [0, 100, 150, 201]):
        o.fill_(7.0)
        op.fwd(q, k, v, torch.tensor(bad, dtype=torch.int32, device="cuda"), o=o)
        assert op.device_status() == -1 and op.device_status() == 0
    _, lse = op.fwd(q, k, v, packed([100, 50, 50]), o=o)
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    for lst, cnt in ([0, 1, 7], 3), ([0, -1, 2], 3), ([0, 1, 2], 4), ([0, 1, 2], -1):
        op.bwd(q, q, k, v, o, lse, packed([100, 50, 50]), alive_in=torch.tensor(lst, dtype=torch.int32, device="cuda"),
               alive_cnt_in=cnt * one)
        assert op.device_status() == -1
    # and the handle still works
    run([100, 50, 50], 2, 2, 64, BF16, False)


@pytest.mark.parametrize("D", [64, 128])
def test_a_wait_that_runs_out_is_reported(D):
    q, k, v = tensors(300, 2, 2, D, BF16, "plain", 15)
    starts = packed([300])
    op = vb.Attention(300, 1, 2, 2, D, BF16)
    good = [x.clone() for x in op.fwd(q, k, v, starts)]
    grads = [x.clone() for x in op.bwd(q, q, k, v, *good, starts)]
    op.set_wait_limit(2_000_000, stall_once=True)
    op.fwd(q, k, v, starts)
    assert op.device_status() == -6
    op.bwd(q, q, k, v, *good, starts)
    assert op.device_status() == -6
    op.set_wait_limit(2_000_000_000)
    again = op.fwd(q, k, v, starts)
    assert all(torch.equal(a, b) for a, b in zip(good, again))
    assert all(torch.equal(a, b) for a, b in zip(grads, op.bwd(q, q, k, v, *good, starts)))
    assert op.device_status() == 0


def test_refusals():
    for kw in (dict(head_dim=12), dict(head_dim=136), dict(heads_kv=3), dict(max_tokens=0), dict(max_seqs=0)):
        with pytest.raises(vb.VcasError):
            vb.Attention(**dict(dict(max_tokens=8, max_seqs=1, heads_q=4, heads_kv=2, head_dim=64), **kw))
    with pytest.raises(ValueError):
        vb.Attention(8, 1, 1, 1, 64, torch.float16)
    op = vb.Attention(8, 1, 2, 2, 64, BF16)
    x = torch.zeros(8, 2, 64, dtype=BF16, device="cuda")
    starts = packed([8])
    with pytest.raises(ValueError):
        op.fwd(x.float(), x, x, starts)
    with pytest.raises(ValueError):
        op.fwd(x, x[:, :1], x, starts)
    with pytest.raises(ValueError):
        op.fwd(x.transpose(1, 2).contiguous().transpose(1, 2), x, x, starts)
    with pytest.raises(ValueError):
        op.fwd(x, x, x, starts, o=x[:1].expand(8, 2, 64))
    with pytest.raises(ValueError):
        op.fwd(x, x, x, starts.long())
    with pytest.raises(ValueError):
        op.fwd(x, x, x, starts.cpu())
    with pytest.raises(ValueError):
        op.bwd(x, x, x, x, x, torch.zeros(2, 8, device="cuda"), starts, alive_in=starts)
    big = torch.zeros(9, 2, 64, dtype=BF16, device="cuda")
    with pytest.raises(vb.VcasError):
        op.fwd(big, big, big, packed([9]))
    with pytest.raises(vb.VcasError):
        op.fwd(x, x, x, packed([4, 4]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [33, 128, 129, 300])
def test_sequences_of_every_length_in_any_number(dtype, causal, n):
    """Tiles are taken in the order of their work while one warp can hold the lengths (128 of them), else as they come."""
    g = torch.Generator().manual_seed(n)
    lens = torch.randint(0, 40, (n,), generator=g).tolist()
    lens[n // 2], lens[3], lens[n - 1] = 400, 260, 129
    run(lens, 2, 1, 64, dtype, causal, "fused")
    alive = sorted(torch.randperm(n, generator=g)[:n - 2].tolist())
    run(lens, 2, 2, 64, dtype, causal, alive=alive)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_broadcast_inputs(dtype):
    """Keys shared by all heads and values shared by all tokens as views with a stride of 0: read as such, gradients for each place."""
    lens, H, D = [150, 33], 3, 64
    T, starts = sum(lens), packed(lens)
    q, k, v = tensors(T, H, H, D, dtype, "plain", 20)
    do = tensors(T, H, H, D, dtype, "plain", 21)[0]
    k, v = k[:, :1].expand(T, H, D), v[:1].expand(T, H, D)
    op = vb.Attention(T, 2, H, H, D, dtype, causal=True)
    ref = reference(q, k, v, starts, True, 0.125, do)
    o, lse = op.fwd(q, k, v, starts)
    check(o, ref["o"], what="o")
    grads = op.bwd(do, q, k, v, ref["o"][0].to(dtype), ref["lse"][0].float(), starts)
    for name, got in zip(("dq", "dk", "dv"), grads):
        check(got, ref[name], what=name)
    for out in (q[:1].expand(T, H, D), q[:, :1].expand(T, H, D)):
        with pytest.raises(ValueError):
            op.fwd(q, k, v, starts, o=out)


@pytest.mark.parametrize("D", [64, 128])
def test_two_handles_on_two_streams(D):
    """Kernels of two handles in flight together share SMs and TMEM; each gives what it gives alone."""
    lens = [700, 300, 129]
    T, starts = sum(lens), packed(lens)
    jobs = []
    for i in range(2):
        q, k, v = tensors(T, 8, 2, D, BF16, "fused", 30 + i)
        do = tensors(T, 8, 2, D, BF16, "plain", 40 + i)[0]
        op = vb.Attention(T, 3, 8, 2, D, BF16, causal=i == 0)
        o, lse = op.fwd(q, k, v, starts)
        alone = [x.clone() for x in (o, lse, *op.bwd(do, q, k, v, o, lse, starts))]
        jobs.append((op, q, k, v, do, alone, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(10):
        for i, (op, q, k, v, do, _, st) in enumerate(jobs):
            with torch.cuda.stream(st):
                o, lse = op.fwd(q, k, v, starts)
                got[i] = (o, lse, *op.bwd(do, q, k, v, o, lse, starts))
    torch.cuda.synchronize()
    for i, (op, *_, alone, _) in enumerate(jobs):
        assert op.device_status() == 0 and all(torch.equal(a, b) for a, b in zip(alone, got[i]))


def test_score_range_that_a_first_tile_does_not_show():
    """The first keys' scores far below the later ones (more than fp32's exponent away), and far above them."""
    T, D = 400, 64
    for sign in (1.0, -1.0):
        g = torch.Generator("cuda").manual_seed(50)
        q = torch.ones(T, 1, D, device="cuda")
        k = 0.05 * torch.randn(T, 1, D, generator=g, device="cuda")
        k += sign * 20.0 * (torch.arange(T, device="cuda")[:, None, None] >= 130).float()      # scores move by 160 / log 2 bits
        v = torch.randn(T, 1, D, generator=g, device="cuda")
        q, k, v = q.to(BF16), k.to(BF16), v.to(BF16)
        starts = packed([T])
        for causal in (False, True):
            op = vb.Attention(T, 1, 1, 1, D, BF16, causal=causal)
            ref = reference(q, k, v, starts, causal, 0.125)
            o, lse = op.fwd(q, k, v, starts)
            check(o, ref["o"], what="o")
            check(lse, ref["lse"], what="lse")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_one_key_has_no_gradient(dtype, D):
    """A row that sees one key has P = 1 and dS = 0, not what is left of two roundings."""
    T = 37
    q, k, v = tensors(T, 4, 2, D, dtype, "plain", 60)
    do = tensors(T, 4, 2, D, dtype, "plain", 61)[0]
    starts = packed([1] * T)
    for causal in (False, True):
        op = vb.Attention(T, T, 4, 2, D, dtype, causal=causal)
        o, lse = op.fwd(q, k, v, starts)
        dq, dk, dv = op.bwd(do, q, k, v, o, lse, starts)
        assert (dq == 0).all() and (dk == 0).all()
        assert torch.equal(o, v.repeat_interleave(2, 1))
        check(dv, reference(q, k, v, starts, causal, D ** -0.5, do)["dv"], what="dv")
    op = vb.Attention(T, 1, 4, 2, D, dtype, causal=True)
    o, lse = op.fwd(q, k, v, packed([T]))
    assert (op.bwd(do, q, k, v, o, lse, packed([T]))[0][0] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [2, 5, 20, 64, 128])
def test_few_keys_do_not_lose_precision_to_the_stored_output(T, D):
    """delta = rowsum(dO O) carries O's rounding into every dS of a row; rows that see one tile of keys take rowsum(P dP).  In norm:
    the result's own rounding and that of dS, each half a step at most and 0.58 of that on average, 2^-8 0.58 sqrt 2 = 0.0032."""
    starts = packed([T] * 8)
    q, k, v = tensors(8 * T, 4, 2, D, BF16, "plain", 62)
    do = tensors(8 * T, 4, 2, D, BF16, "plain", 63)[0]
    for causal in (False, True):
        op = vb.Attention(8 * T, 8, 4, 2, D, BF16, causal=causal)
        o, lse = op.fwd(q, k, v, starts)
        grads = op.bwd(do, q, k, v, o, lse, starts)
        ref = reference(q, k, v, starts, causal, D ** -0.5, do)
        for name, got in zip(("dq", "dk", "dv"), grads):
            want = ref[name][0]
            assert float((got.double() - want).norm() / want.norm()) <= 0.0032, name


@pytest.mark.parametrize("D", [40, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Hq,Hk", [(2, 2), (4, 1), (3, 1)])
def test_rows_of_few_keys_have_the_rounding_of_their_result_alone(D, causal, Hq, Hk):
    lens = [1, 2, 3, 17, 40, 63, 64]
    starts = packed(lens)
    total = sum(lens)
    q, k, v = tensors(total, Hq, Hk, D, BF16, "plain", 3)
    do = tensors(total, Hq, Hk, D, BF16, "plain", 4)[0]
    op = vb.Attention(total, len(lens), Hq, Hk, D, BF16, causal=causal)
    ref = reference(q, k, v, starts, causal, 1.0 / math.sqrt(D), do, parts=2)
    o, lse = op.fwd(q, k, v, starts)
    check(o, ref["o"], what="o")
    grads = op.bwd(do, q, k, v, ref["o"][0].to(BF16), ref["lse"][0].float(), starts)
    for name, x in zip(("dq", "dk", "dv"), grads):
        check(x, ref[name], what=name)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [8, 40, 72, 128])
@pytest.mark.parametrize("layout", ["plain", "heads", "odd"])
def test_rows_of_dropped_sequences_become_zero_in_every_layout(dtype, D, layout):
    lens = [(37 * i * i) % 91 for i in range(40)]        # some empty
    run(lens, 6, 2, D, dtype, False, layout, alive=list(range(1, 40, 3)), behind=3)


@pytest.mark.parametrize("dtype,D", [(F32, 64), (BF16, 64), (BF16, 128)])
def test_offsets_beyond_32_bits(dtype, D):
    """Tokens 2^23 elements apart, 2.5e9 elements from the first to the last: the same bits as side by side."""
    lens, Hq, Hk, far = [100, 130, 70], 4, 2, 1 << 23
    starts, total = packed(lens), sum(lens)
    store = torch.empty(total * far, dtype=dtype, device="cuda")
    place = [0]

    def apart(h, like=None):
        x = torch.as_strided(store, (total, h, D), (far, D, 1), place[0])
        place[0] += h * D
        return x if like is None else x.copy_(like)

    q, k, v = tensors(total, Hq, Hk, D, dtype, "plain", 5)
    do = tensors(total, Hq, Hk, D, dtype, "plain", 6)[0]
    op = vb.Attention(total, 3, Hq, Hk, D, dtype, causal=True)
    o, lse = op.fwd(q, k, v, starts)
    kept = dict(alive_in=torch.tensor([1, 2, 0], dtype=torch.int32, device="cuda"), alive_cnt_in=torch.tensor([2], dtype=torch.int32, device="cuda"))
    want = op.bwd(do, q, k, v, o, lse, starts, **kept)
    q2, k2, v2, do2 = apart(Hq, q), apart(Hk, k), apart(Hk, v), apart(Hq, do)
    o2, lse2 = op.fwd(q2, k2, v2, starts, o=apart(Hq))
    got = op.bwd(do2, q2, k2, v2, o2, lse2, starts, dq=apart(Hq), dk=apart(Hk), dv=apart(Hk), **kept)
    assert op.device_status() == 0
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [4, 200])
def test_a_list_that_does_not_ascend_is_reported(dtype, n):
    """The same sequence twice: the second entry is left out and reported, the others' results are those of the list without it."""
    lens = [33 + 7 * (i % 5) for i in range(n)]
    starts, total = packed(lens), sum(lens)
    q, k, v = tensors(total, 2, 1, 64, dtype, "plain", 8)
    do = tensors(total, 2, 1, 64, dtype, "plain", 9)[0]
    op = vb.Attention(total, n, 2, 1, 64, dtype, causal=True)
    o, lse = op.fwd(q, k, v, starts)
    lst = lambda x: dict(alive_in=torch.tensor(x + [0] * (n - len(x)), dtype=torch.int32, device="cuda"),
                         alive_cnt_in=torch.tensor([len(x)], dtype=torch.int32, device="cuda"))
    want = op.bwd(do, q, k, v, o, lse, starts, **lst([1, n - 1]))
    assert op.device_status() == 0
    got = op.bwd(do, q, k, v, o, lse, starts, **lst([1, 1, n - 1]))
    assert op.device_status() == -1
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    op.bwd(do, q, k, v, o, lse, starts, **lst([n - 1, 1]))
    assert op.device_status() == -1 and op.device_status() == 0
