"""The AdamW step against its formulas: every operation rounded to fp32 on its own, so that with fp32 states results are the same to
the bit, and 8-bit states are one of the two neighbours that the random bits choose between."""
import math

import numpy as np
import pytest
import torch

from paper_2402_17227_b200 import binding as vb

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
LR, B1, B2, EPS = 1e-3, 0.9, 0.999, 1e-8


def f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def step_32(p, g, m, v, step, wd, scale=1.0):
    """One step in numpy's fp32, whose operations are each rounded by themselves (torch's on the CPU differ in a last bit now and then)."""
    f = lambda x: np.float32(x)
    step_size, inv = f(LR / (1.0 - B1 ** step)), f(1.0 / math.sqrt(1.0 - B2 ** step))
    p, g, m, v = (t.float().numpy() for t in (p, g, m, v))
    g = g * f(scale)
    m = m * f(B1) + g * f(1.0 - B1)
    v = v * f(B2) + (g * g) * f(1.0 - B2)
    root = np.sqrt(v)
    p = p * f(1.0 - LR * float(f(wd))) - (m * step_size) / (root * inv + f(EPS))
    return tuple(torch.from_numpy(x) for x in (p, m, v, root))


def tensor(n, dtype, off, seed, device="cuda", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.zeros(n + off, dtype=dtype, device=device)
    x[off:] = (scale * torch.randn(n, generator=g)).to(dtype).to(device)
    return x[off:]


SIZES = [0, 1, 7, 8, 255, 256, 257, 2048, 2049, 5000, 100003]


@pytest.mark.parametrize("pd", [F32, BF16])
@pytest.mark.parametrize("gd", [F32, BF16])
@pytest.mark.parametrize("off", [0, 1])
def test_32_bit_states_to_the_bit(pd, gd, off):
    entries, want = [], []
    for i, n in enumerate(SIZES):
        p, g = tensor(n, pd, off, 10 * i), tensor(n, gd, off, 10 * i + 1, scale=10.0 ** (i % 5 - 3))
        m, v = tensor(n, F32, off, 10 * i + 2), tensor(n, F32, off, 10 * i + 3).abs_()
        if n > 20:
            g[3:9] = 0
            m[3:9] = 0
            v[3:9] = 0
        copy = tensor(n, BF16, off, 5) if pd == F32 and i % 2 else None
        wd = 0.1 * (i % 3)
        entries.append(vb.AdamWTensor(p, g, m, v, copy=copy, weight_decay=wd))
        want.append(step_32(*[t.cpu() for t in (p, g, m, v)], 3, wd))
    vb.AdamW(entries).step(3, lr=LR, beta1=B1, beta2=B2, eps=EPS)
    for e, (p, m, v, _) in zip(entries, want):
        assert torch.equal(e.p.cpu(), p.to(pd)) and torch.equal(e.m.cpu(), m) and torch.equal(e.v.cpu(), v)
        if e.copy is not None:
            assert torch.equal(e.copy.cpu(), p.to(BF16))


def values(codes, scale):
    n = codes.numel()
    return codes.cpu().float() * scale.cpu().repeat_interleave(256)[:n]


def eight_bit(n, off, seed, pd=F32, gd=F32, copy=True):
    e = vb.AdamWTensor.make(tensor(n, pd, off, seed), tensor(n, gd, off, seed + 1, scale=1e-3), 8,
                            copy=tensor(n, BF16, off, 5) if copy and pd == F32 else None, weight_decay=0.01)
    if off:
        e.m, e.v = (torch.zeros(n + off, dtype=torch.uint8, device="cuda").view(E4M3)[off:] for _ in range(2))
    return e


@pytest.mark.parametrize("pd", [F32, BF16])
@pytest.mark.parametrize("gd", [F32, BF16])
@pytest.mark.parametrize("off", [0, 1])
def test_8_bit_states(pd, gd, off):
    """Several steps: p from the states held before the step; each new state is an e4m3 neighbour of the exact value.  The
    quotient is good to 2^-22 and the root to a rounding: the update to 2^-21, with a rounding of p behind it."""
    entries = [eight_bit(n, off, 20 * i, pd, gd) for i, n in enumerate(SIZES)]
    grid = torch.arange(127, dtype=torch.uint8).view(E4M3).float()            # 0 .. 448, ascending
    opt = vb.AdamW(entries)
    for step in range(1, 5):
        before = [(e.p.cpu().clone(), e.g.cpu().clone(), values(e.m, e.m_scale), values(e.v, e.v_scale)) for e in entries]
        opt.step(step, lr=LR, beta1=B1, beta2=B2, eps=EPS, seed=step)
        for e, (p, g, m, r) in zip(entries, before):
            wp, wm, _, wr = step_32(p, g, m, r * r, step, 0.01)
            n = wp.numel()
            off_by = 2.0 ** -21 * (wp - p.float() * f32(1.0 - LR * f32(0.01))).abs() + 2.0 ** -23 * wp.abs()
            u = torch.finfo(pd).eps / 2
            assert ((e.p.cpu().float() - wp).abs() <= off_by * (1 + 2 * u) + (u * 1.01 * wp.abs() if pd == BF16 else 0)).all()
            if e.copy is not None:
                assert torch.equal(e.copy, e.p.to(BF16))
            for codes, scale, want, least in ((e.m, e.m_scale, wm, 0), (e.v, e.v_scale, wr, 1)):
                if n == 0:
                    continue
                pad = torch.zeros((n + 255) // 256 * 256)
                pad[:n] = want.abs()
                big = pad.view(-1, 256).amax(1)
                assert ((scale.cpu() - big * f32(1 / 448)).abs() <= (2.0 ** -21 if least else 0) * scale.cpu()).all()
                y = torch.where(big > 0, 448.0 / big, torch.zeros(()))[:, None] * pad.view(-1, 256)
                y = y.reshape(-1)[:n].clamp_max(448.0)
                c = codes.cpu().float()
                assert torch.equal(torch.sign(c) * (c != 0), torch.sign(want) * (c != 0))
                at = torch.searchsorted(grid, y, right=True) - 1               # the neighbour below
                below, above = grid[at], grid[(at + 1).clamp_max(126)]
                # 448 / big, its product and the value itself (2^-22 where it is a root): y may lie that close to a neighbour
                tie = (y - below).abs() <= 2.0 ** -20 * y
                tie |= (above - y).abs() <= 2.0 ** -20 * y
                ok = (c.abs() == below) | (c.abs() == above) | tie
                ok |= (least == 1) & (y > 0) & (c == grid[1])
                assert ok.all()
                if least:
                    assert ((c > 0) == (want > 0)).all()


def test_rounding_is_unbiased_and_follows_the_seed():
    """With g = 0 and beta1 = 0.9, m shrinks to 0.9 of itself: between two e4m3 values, on average by exactly that."""
    n = 256 * 512
    grad = torch.zeros(n, device="cuda")
    grad[::256] = 448.0
    e = vb.AdamWTensor.make(torch.zeros(n, device="cuda"), grad, 8)
    e.m.view(torch.uint8).fill_(0x38)                 # 1.0
    e.m.view(torch.uint8)[::256] = 0x7E               # 448, which its gradient of 448 keeps there, and the scale at 1
    e.m_scale.fill_(1.0)
    other = vb.AdamWTensor(e.p.clone(), e.g, e.m.view(torch.uint8).clone().view(E4M3), e.v.view(torch.uint8).clone().view(E4M3),
                           e.m_scale.clone(), e.v_scale.clone())
    vb.AdamW([e]).step(1, lr=0.0, seed=1)
    vb.AdamW([other]).step(1, lr=0.0, seed=2)
    got = values(e.m, e.m_scale)
    small = torch.ones(n, dtype=torch.bool)
    small[::256] = False
    lo, hi = got[small].min(), got[small].max()
    share = float((got[small] == hi).double().mean())
    # 0.9 lies between two neighbours w apart; the mean of 130560 draws is within 5 standard deviations, and 1/512 for the 8 bits
    w = float(hi - lo)
    assert abs(lo - 0.875) < 1e-5 and abs(hi - 0.9375) < 1e-5 and abs(float(got[small].double().mean()) - 0.9) <= w * (5 * math.sqrt(share * (1 - share) / small.sum()) + 1 / 512)
    assert not torch.equal(e.m.view(torch.uint8), other.m.view(torch.uint8))
    again = vb.AdamWTensor.make(torch.zeros(n, device="cuda"), grad, 8)
    again.m.view(torch.uint8).fill_(0x38)
    again.m.view(torch.uint8)[::256] = 0x7E
    again.m_scale.fill_(1.0)
    vb.AdamW([again]).step(1, lr=0.0, seed=1)
    assert torch.equal(e.m.view(torch.uint8), again.m.view(torch.uint8))


def test_a_state_that_moves_by_less_than_a_step_still_moves():
    """r = sqrt(v) changes by under 0.1 % a step, an e4m3 step is 6 to 12 %: over 400 steps it has to arrive all the same."""
    n = 256 * 16
    e = vb.AdamWTensor.make(torch.zeros(n, device="cuda"), torch.full((n,), 0.5, device="cuda"), 8)
    e.v.view(torch.uint8).fill_(0x7E)
    e.v_scale.fill_(1.0 / 448.0)                      # r = 1; gradients of 0.5 pull it towards 0.5
    opt = vb.AdamW([e])
    for s in range(1, 401):
        opt.step(s, lr=0.0, seed=s)
    r = values(e.v, e.v_scale).double()
    want = math.sqrt(0.25 + 0.75 * B2 ** 400)         # 0.868
    # the block's scale follows its largest value, whose random rounding goes up as often as down: a few per cent are left
    assert abs(float(r.pow(2).mean().sqrt()) - want) < 0.05


def test_many_tensors_more_than_one_launch_holds():
    entries = [vb.AdamWTensor.make(tensor(100 + i, F32, 0, i), tensor(100 + i, F32, 0, 1000 + i), 8 if i % 3 == 0 else 32, weight_decay=0.01)
               for i in range(1300)]
    want = [step_32(e.p.cpu(), e.g.cpu(), torch.zeros(e.p.numel()), torch.zeros(e.p.numel()), 1, 0.01)[0] for e in entries]
    before = [e.p.cpu() for e in entries]
    vb.AdamW(entries).step(1, lr=LR)
    for e, w, b in zip(entries, want, before):       # 8-bit states: update to 2^-21, and a rounding
        near = (2.0 ** -21 * (w - b).abs() + 2.0 ** -23 * w.abs()) if e.m.dtype == E4M3 else torch.zeros(())
        assert ((e.p.cpu() - w).abs() <= near).all()


def test_nan_gradients_stay_where_they_belong():
    for bits in (8, 32):
        e = vb.AdamWTensor.make(tensor(1000, F32, 0, 1), tensor(1000, F32, 0, 2), bits)
        clean = vb.AdamWTensor.make(e.p.clone(), e.g.clone(), bits)
        e.g[300] = float("nan")
        for x in (e, clean):
            vb.AdamW([x]).step(1, lr=LR, seed=3)
        rest = torch.arange(1000) != 300
        assert e.p[300].isnan() and torch.equal(e.p.cpu()[rest], clean.p.cpu()[rest])
        if bits == 8:
            assert e.m_scale[1].isnan() and torch.equal(e.m_scale[[0, 2, 3]], clean.m_scale[[0, 2, 3]])
            block = (torch.arange(1000) // 256 == 1)
            assert torch.equal(e.m.view(torch.uint8).cpu()[~block], clean.m.view(torch.uint8).cpu()[~block])


def test_device_scalars_and_a_captured_step():
    """grad_scale, rates and seed on the device: a replayed step follows them, and is the step with the host's numbers."""
    for bits in (32, 8):
        make = lambda: vb.AdamWTensor.make(tensor(3000, F32, 0, 4), tensor(3000, BF16, 0, 5, scale=0.1), bits, weight_decay=0.5)
        a, b = make(), make()
        scale = torch.tensor([0.25], device="cuda")
        rates, seed = torch.zeros(3, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        opt = vb.AdamW([a])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            opt.step(1, lr=0.0, grad_scale=scale, rates=rates, seed_dev=seed)
        for s in (1, 2, 3):
            lr = 2.0 ** -s                            # exact in fp32, so that both ways decay by the same factor
            rates.copy_(vb.adamw_rates(lr, 0.9, 0.999, s))
            seed.fill_(s)
            scale.fill_(1.0 / s)
            graph.replay()
            vb.AdamW([b]).step(s, lr=lr, seed=s, grad_scale=scale)
            torch.cuda.synchronize()
            for x, y in ((a.p, b.p), (a.m.view(torch.uint8), b.m.view(torch.uint8)), (a.v.view(torch.uint8), b.v.view(torch.uint8))):
                assert torch.equal(x, y)
        del graph


def test_refusals():
    p, g = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    z = lambda n, dt=F32: torch.zeros(n, dtype=dt, device="cuda")
    e8 = z(300, torch.uint8).view(E4M3)
    for bad in (lambda: vb.AdamWTensor(p, g, z(299), z(300)), lambda: vb.AdamWTensor(p.half(), g, z(300), z(300)),
                lambda: vb.AdamWTensor(p, g.double(), z(300), z(300)), lambda: vb.AdamWTensor(p, g[:299], z(300), z(300)),
                lambda: vb.AdamWTensor(p, g, e8, e8), lambda: vb.AdamWTensor(p, g, e8, e8, z(1), z(2)),
                lambda: vb.AdamWTensor(p, g, z(300), z(300), z(2), z(2)), lambda: vb.AdamWTensor(p, g, e8, z(300)),
                lambda: vb.AdamWTensor(p, g, z(300), z(300), copy=z(300)),
                lambda: vb.AdamWTensor(p.bfloat16(), g, z(300), z(300), copy=z(300, BF16)),
                lambda: vb.AdamWTensor(p[::2], g[:150], z(150), z(150)), lambda: vb.AdamWTensor(p.cpu(), g, z(300), z(300))):
        with pytest.raises(ValueError):
            vb.AdamW([bad()])
    good = vb.AdamW([vb.AdamWTensor.make(p, g)])
    for kw in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(lr=-1.0), dict(lr=float("nan")), dict(eps=-1.0)):
        with pytest.raises(vb.VcasError):
            good.step(**dict(dict(step=1, lr=LR), **kw))
    with pytest.raises(vb.VcasError):
        vb.AdamW([vb.AdamWTensor.make(p, g, weight_decay=-1.0)]).step(1, lr=LR)
    with pytest.raises(ValueError):
        good.step(1, lr=LR, grad_scale=torch.ones(1))
    vb.AdamW([]).step(1, lr=LR)


@pytest.mark.parametrize("eps", [0.0, 1e-40])
def test_8_bit_states_of_the_smallest_gradients(eps):
    """v = (1 - beta2) g^2 under fp32's normal numbers counts as 2^-126, eps (not 0) as no less: the step is finite and that of the formula
    with them.  Four roundings, an ulp each of root and reciprocal: 2^-20 relative is more than all.  Without a gradient p stays."""
    n = 512
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 1e-20, device="cuda")
    p[256:], g[256:] = 1.0, 0.0
    t = vb.AdamWTensor.make(p, g, bits=8)
    vb.AdamW([t]).step(1, lr=LR, beta1=B1, beta2=B2, eps=eps)
    m = (1.0 - B1) * 1e-20
    denom = 2.0 ** -63 / math.sqrt(1.0 - B2) + (2.0 ** -126 if eps else 0.0)
    want = -LR / (1.0 - B1) * m / denom
    assert ((p[:256].double() / want - 1.0).abs() <= 2.0 ** -20).all()
    if eps:
        assert (p[256:] == 1.0).all()
    r = t.v.float() * t.v_scale.repeat_interleave(256)
    assert (r[256:] == 0).all() and ((r[:256].double() / 2.0 ** -63 - 1.0).abs() <= 2.0 ** -20).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_more_elements_than_31_bits_count(bits):
    """The last elements of 2^31 + 4864 get the step that they get in a tensor of their own."""
    n, few = (1 << 31) + 4864, 4864
    p, g = torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    p[-few:], g[-few:] = tensor(few, BF16, 0, 1), tensor(few, BF16, 0, 2, scale=1e-2)
    small, large = (vb.AdamWTensor.make(p[-few:].clone(), g[-few:].clone(), bits, weight_decay=0.1),
                    vb.AdamWTensor.make(p, g, bits, weight_decay=0.1))
    vb.AdamW([small]).step(2, lr=LR, beta1=B1, beta2=B2, eps=EPS, seed=3)
    vb.AdamW([large]).step(2, lr=LR, beta1=B1, beta2=B2, eps=EPS, seed=3)
    assert torch.equal(large.p[-few:], small.p)
    if bits == 32:
        assert torch.equal(large.m[-few:], small.m) and torch.equal(large.v[-few:], small.v)
    else:
        assert torch.equal(large.m_scale[-few // 256:], small.m_scale) and torch.equal(large.v_scale[-few // 256:], small.v_scale)
    assert (large.p[:-few].view(torch.int32) == 0).all()
