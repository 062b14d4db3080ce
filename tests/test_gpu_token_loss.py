"""Log probabilities of given tokens, entropy, top alternatives and their gradient against 64-bit formulas."""
import pytest
import torch

from paper_2402_17227_b200 import binding as vb

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
F = 2.0 ** -24


def logits_of(rows, vocab, dtype, pad=0, off=0, seed=0, scale=3.0):
    """[rows, vocab] whose rows start `off` elements behind a 16-byte boundary and have `pad` unused columns of NaN behind them."""
    g = torch.Generator("cuda").manual_seed(seed)
    store = torch.full((rows * (vocab + pad) + off + 8,), float("nan"), dtype=dtype, device="cuda")
    x = store[off:off + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    x.copy_((scale * torch.randn(rows, vocab, generator=g, device="cuda")).to(dtype))
    return x


def tokens_of(rows, vocab, seed=1, dtype=torch.int64):
    g = torch.Generator("cuda").manual_seed(seed)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    t[torch.rand(rows, generator=g, device="cuda") < 0.2] = -1
    return t.to(dtype)


def formulas(x, tokens, top):
    """lse, logp, entropy, the top ids and their log probabilities in 64 bits; a row of -inf has no distribution."""
    x = x.double()
    none = (x == float("-inf")).all(1)
    m = x.amax(1, keepdim=True)
    lse = torch.logsumexp(x, 1)
    lp = torch.where(none[:, None], float("-inf"), (x - m) - torch.log(torch.exp(x - m).sum(1, keepdim=True)))
    p = torch.where(none[:, None], 0.0, lp.exp())
    H = -torch.where(p > 0, p * lp, 0.0).sum(1)
    has = tokens >= 0
    given = torch.where(has, lp.gather(1, tokens.long().clamp_min(0)[:, None])[:, 0], 0.0)
    ids = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :top].int()
    return lse, given, H, ids, lp.gather(1, ids.long()), lp, p


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    same = (got == want) | ((got - want).abs() <= bound) | (got.isnan() & want.isnan())
    assert same.all(), (what, float((got - want).abs()[~same].max()))


def errors(x, lp, p, H, vocab):
    """What fp32 may lose.  d = x - max has half a step of |d|; exp of it 2^-21 (its own error) + 2 F |d| (argument); sums of n terms
    n / threads + log2(threads) roundings, taken as n F at most 64 F.  lse and logp add a rounding of their size."""
    n = min(vocab, 64)
    d = torch.where(p > 0, -lp, 0.0)                  # |x - lse|, as large as |x - max| up to log(n)
    e_sum = 2.0 ** -21 + n * F + 3 * F * (p * d).sum(1)
    e_ent = (p * d * (2.0 ** -20 + (n + 6) * F + 3 * F * d)).sum(1) + e_sum * (1 + H.abs()) + 4 * F * H.abs()
    return e_sum, e_ent


def run_fwd(x, tokens, top):
    op = vb.TokenLoss(x.shape[0], x.shape[1], x.dtype, top=top)
    r = op.fwd(x, tokens)
    assert op.device_status() == 0
    op.close()
    return r


def check_fwd(x, tokens, top):
    r = run_fwd(x, tokens, top)
    lse, given, H, ids, top_lp, lp, p = formulas(x, tokens, max(top, 1))
    e_sum, e_ent = errors(x, lp, p, H, x.shape[1])
    close(r.lse, lse, e_sum + 2 * F * lse.abs().nan_to_num(0, 0, 0), "lse")
    close(r.logp, given, e_sum + 4 * F * given.abs().nan_to_num(0, 0, 0), "logp")
    close(r.entropy, H, e_ent, "entropy")
    if top:
        assert torch.equal(r.top_ids, ids)
        close(r.top_logp, top_lp, (e_sum[:, None] + 4 * F * top_lp.abs().nan_to_num(0, 0, 0)), "top_logp")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [1, 5, 32, 50, 257, 1000, 1025, 4099, 32000, 70001])
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_forward_sizes(dtype, vocab, rows):
    x = logits_of(rows, vocab, dtype, pad=3, off=1, seed=vocab + rows)
    check_fwd(x, tokens_of(rows, vocab), min(20, vocab))
    check_fwd(x, tokens_of(rows, vocab, dtype=torch.int32), 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("off", range(8))
def test_forward_any_alignment(dtype, off):
    check_fwd(logits_of(70, 555, dtype, pad=off, off=off, seed=off), tokens_of(70, 555), 7)
    check_fwd(logits_of(2, 30011, dtype, pad=off, off=off, seed=off), tokens_of(2, 30011), 32)


@pytest.mark.parametrize("rows", [2, 700])
@pytest.mark.parametrize("top", [1, 2, 31, 32])
def test_many_rows_and_every_top(rows, top):
    check_fwd(logits_of(rows, 5000, BF16, seed=top), tokens_of(rows, 5000), top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [40, 3001, 50000])
def test_ties_order_and_hard_rows(dtype, vocab):
    """Equal values (the lowest index first), ascending and descending rows, all large values in one thread's hands, -0 and 0."""
    x = logits_of(8, vocab, dtype, seed=2)
    i = torch.arange(vocab, device="cuda", dtype=torch.float32)
    x[0] = 1.5
    x[1] = (i / vocab * 4 - 2).to(dtype)
    x[2] = (2 - i / vocab * 4).to(dtype)
    x[3] = torch.where((i.long() // 8) % 256 == 3, 5.0 + (i % 97) / 97, 0.0).to(dtype)
    x[4] = torch.where(i.long() % 2 == 0, 0.0, -0.0).to(dtype)
    x[5] = torch.where(i < 20, 3.0, -1.0).to(dtype)
    x[6] = torch.where(i >= vocab - 9, 3.0, -1.0).to(dtype)
    check_fwd(x, tokens_of(8, vocab), 20)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [33, 2500, 40000])
def test_masked_rows(dtype, vocab):
    """-inf, the type's lowest value, rows with one value or none left, logits far from 0."""
    lowest = torch.finfo(dtype).min
    x = logits_of(9, vocab, dtype, seed=4)
    x[0] = float("-inf")
    x[1, 1:] = float("-inf")
    x[2] = lowest
    x[3, :-1] = lowest
    x[4, ::2] = float("-inf")
    x[5] += 20000.0
    x[6] -= 20000.0
    x[7, 3:] = lowest
    x[7, 5:] = float("-inf")
    x[8, :vocab // 2] = float("-inf")
    t = tokens_of(9, vocab)
    t[:9] = torch.tensor([3, 0, 1, vocab - 1, 1, 2, 3, 0, vocab - 1], device="cuda")
    check_fwd(x, t, 5)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("vocab", [60, 9000])
def test_nan_and_infinity_stay_in_their_row(bad, vocab):
    for dtype in (F32, BF16):
        x = logits_of(3, vocab, dtype, seed=6)
        clean = run_fwd(x, tokens_of(3, vocab).abs(), 4)
        x[1, vocab // 3] = bad
        r = run_fwd(x, tokens_of(3, vocab).abs(), 4)
        for a, b in zip((r.lse, r.logp, r.entropy, r.top_logp, r.top_ids), (clean.lse, clean.logp, clean.entropy, clean.top_logp, clean.top_ids)):
            assert torch.equal(a[[0, 2]], b[[0, 2]])
        assert r.lse[1].isnan() and r.logp[1].isnan() and r.entropy[1].isnan() and r.top_logp[1].isnan().all()
        assert ((r.top_ids[1] >= -1) & (r.top_ids[1] < vocab)).all()


def backward_of(x, tokens, lse, H, gl, ge):
    x, gl = x.double(), torch.where(tokens >= 0, gl.double(), 0.0)
    none = lse == float("-inf")
    lp = torch.where(none[:, None], -1e30, x - lse.double()[:, None])
    p = lp.exp()
    onehot = torch.zeros_like(p).scatter_(1, tokens.long().clamp_min(0)[:, None], 1.0)
    d = torch.where(none[:, None], 0.0, gl[:, None] * (onehot - p))
    mag = gl.abs()[:, None] * (onehot + p)
    if ge is not None:
        t = torch.where(p > 0, ge.double()[:, None] * p * (lp + H.double()[:, None]), 0.0)
        d = d - t
        mag = mag + ge.double().abs()[:, None] * p * torch.where(p > 0, lp.abs() + H.double().abs()[:, None], 0.0)
    return d, mag, torch.where(p > 0, lp.abs(), 0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab,pad,off", [(1, 0, 0), (7, 2, 1), (50, 0, 3), (1000, 0, 0), (4099, 5, 7), (32000, 0, 0)])
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("rows", [2, 600])
def test_backward(dtype, vocab, pad, off, entropy, rows):
    x = logits_of(rows, vocab, dtype, pad, off, seed=vocab)
    if vocab > 20:
        x[:, 5:11] = float("-inf")
        x[1] = float("-inf")
    tokens = tokens_of(rows, vocab)
    lse, _, H, *_ = formulas(x, tokens, 1)
    lse, H = lse.float(), H.float()
    g = torch.Generator("cuda").manual_seed(8)
    gl = torch.randn(rows, generator=g, device="cuda")
    gl[tokens < 0] = float("nan")                       # nothing flows through a row without a token
    ge = torch.randn(rows, generator=g, device="cuda") if entropy else None
    op = vb.TokenLoss(rows, vocab, dtype)
    out = logits_of(rows, vocab, dtype, pad + 1, off, seed=9)
    mark = out.storage_offset()
    for d in (out, None):
        d, norms = op.bwd(x, tokens, lse, gl, entropy=H if entropy else None, g_entropy=ge, dlogits=d)
        want, mag, depth = backward_of(x, tokens, lse, H, gl.nan_to_num(0), ge)
        u = torch.finfo(dtype).eps / 2
        # exp: 2^-21, its argument 2 F |log p|; five fp32 operations; one rounding of what is stored (or the type's smallest step)
        bound = mag * (2.0 ** -20 + (8 + 3 * depth) * F) + 1.01 * u * want.abs() + torch.finfo(dtype).tiny
        close(d, want, bound, "dlogits")
        sq = d.double().square().sum(1)
        close(norms, sq, sq * (min(vocab, 64) + 16) * F + 1e-37, "row norms")
    same = x.clone()
    op2 = op.bwd(same, tokens, lse, gl, entropy=H if entropy else None, g_entropy=ge, dlogits=same)[0]
    assert torch.equal(op2, d) and op2.data_ptr() == same.data_ptr() and mark == out.storage_offset()
    assert op.device_status() == 0
    op.close()


def test_gradient_against_differences():
    rows, vocab = 4, 300
    x = logits_of(rows, vocab, F32, seed=10)
    tokens = tokens_of(rows, vocab).abs()
    g = torch.Generator("cuda").manual_seed(11)
    gl, ge = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    op = vb.TokenLoss(rows, vocab, F32)
    r = op.fwd(x, tokens)
    d, _ = op.bwd(x, tokens, r.lse, gl, entropy=r.entropy, g_entropy=ge)
    way = torch.randn(rows, vocab, generator=g, device="cuda", dtype=torch.float64)

    def loss(z):
        _, given, H, *_ = formulas(z, tokens, 1)
        return float((gl.double() * given + ge.double() * H).sum())

    h = 1e-5
    diff = (loss(x.double() + h * way) - loss(x.double() - h * way)) / (2 * h)
    # central difference: h^2 / 6 of the third derivative (below 1e-8 here); fp32 gradient: about 1e-6 of its size
    assert abs(float((d.double() * way).sum()) - diff) <= 1e-5 * float((d.double() * way).abs().sum())


def test_a_token_outside_the_vocabulary_is_reported():
    x = logits_of(3, 40, F32)
    op = vb.TokenLoss(3, 40, F32)
    t = torch.tensor([1, 40, -7], device="cuda")
    r = op.fwd(x, t)
    assert op.device_status() == -1 and op.device_status() == 0
    assert r.logp[1] == 0 and r.logp[2] == 0 and r.logp[0] < 0
    d, n = op.bwd(x, t, r.lse, torch.ones(3, device="cuda"))
    assert op.device_status() == -1 and (d[1:] == 0).all() and (n[1:] == 0).all() and n[0] > 0


def test_captured_and_on_another_stream():
    x, t = logits_of(5, 20000, BF16, seed=12), tokens_of(5, 20000)
    op = vb.TokenLoss(5, 20000, BF16, top=5)
    first = op.fwd(x, t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = op.fwd(x, t)
    torch.cuda.current_stream().wait_stream(side)
    for n in ("lse", "logp", "entropy", "top_logp", "top_ids"):
        assert torch.equal(getattr(first, n), getattr(again, n))
    graph = torch.cuda.CUDAGraph()
    gl = torch.ones(5, device="cuda")
    with torch.cuda.graph(graph):
        r = op.fwd(x, t)
        d, norms = op.bwd(x, t, r.lse, gl)
    x.copy_(logits_of(5, 20000, BF16, seed=13))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    want = run_fwd(x, t, 5)
    assert torch.equal(r.lse, want.lse) and torch.equal(r.top_ids, want.top_ids)
    assert torch.equal(norms, op.bwd(x, t, r.lse, gl)[1])
    del graph


def test_no_rows():
    op = vb.TokenLoss(4, 50, F32, top=3)
    r = op.fwd(torch.zeros(0, 50, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"))
    assert r.lse.numel() == 0 and r.top_ids.shape == (0, 3)


def test_refusals():
    for kw in (dict(vocab=0), dict(max_rows=0), dict(top=33), dict(vocab=10, top=11), dict(top=-1)):
        with pytest.raises(vb.VcasError):
            vb.TokenLoss(**dict(dict(max_rows=4, vocab=50, dtype=F32, top=0), **kw))
    with pytest.raises(ValueError):
        vb.TokenLoss(4, 50, torch.float16)
    op = vb.TokenLoss(4, 50, F32)
    x, t, v = torch.zeros(4, 50, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    for bad in (lambda: op.fwd(x.bfloat16(), t), lambda: op.fwd(x[:, :49], t), lambda: op.fwd(x, t[:3]), lambda: op.fwd(x, t.float()),
                lambda: op.fwd(x.t().contiguous().t(), t), lambda: op.fwd(x, t.cpu()), lambda: op.fwd(x[:1].expand(4, 50), t),
                lambda: op.bwd(x, t, v[:3], v), lambda: op.bwd(x, t, v, v.double())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(vb.VcasError):
        op.fwd(torch.zeros(5, 50, device="cuda"), torch.zeros(5, dtype=torch.int64, device="cuda"))
    with pytest.raises(vb.VcasError):
        op.bwd(x, t, v, v, g_entropy=v)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_offsets_beyond_32_bits(dtype):
    """Rows 2^24 elements apart, 2.3e9 elements from the first to the last: the same bits as side by side."""
    rows, vocab, far = 140, 1000, 1 << 24
    x = logits_of(rows, vocab, dtype, pad=8)
    tokens = tokens_of(rows, vocab)
    op = vb.TokenLoss(rows, vocab, dtype, top=5)
    apart = lambda at: torch.as_strided(store, (rows, vocab), (far, 1), at)
    store = torch.empty(rows * far, dtype=dtype, device="cuda")
    y = apart(0).copy_(x)
    a, b = op.fwd(x, tokens), op.fwd(y, tokens)
    for name in ("logp", "entropy", "lse", "top_logp", "top_ids"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    g = -torch.rand(rows, device="cuda")
    want = op.bwd(x, tokens, a.lse, g, entropy=a.entropy, g_entropy=0.1 * g)
    got = op.bwd(y, tokens, a.lse, g, entropy=a.entropy, g_entropy=0.1 * g, dlogits=apart(4096))
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
