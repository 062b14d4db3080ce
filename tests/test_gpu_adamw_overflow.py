"""AdamW where a finite gradient's square leaves fp32's range: v is infinite, m / sqrt(v) is 0, and p only decays, with states of
either width."""
import pytest
import torch

from paper_2402_17227_b200 import binding as vb
from tests.test_gpu_adamw import B1, B2, BF16, E4M3, EPS, F32, LR, f32, tensor

pytestmark = pytest.mark.gpu
N, AT = 1000, [0, 300, 301, 999]              # of four blocks the first, the second (twice) and the last


@pytest.mark.parametrize("pd", [F32, BF16])
@pytest.mark.parametrize("gd", [F32, BF16])
@pytest.mark.parametrize("big", [2e19, 1e21, -1e21, 3e38])
def test_p_decays_and_nothing_else_is_lost(pd, gd, big):
    """Exact: p (1 - lr wd), rounded once, is what both widths give where v is infinite.  The other elements' p comes from the states before
    the step, which no neighbour touches."""
    steps, keep = {}, f32(1.0 - LR * f32(0.1))
    for bits in (32, 8):
        for spoil in (False, True):
            g = tensor(N, gd, 0, 2, scale=1e-2)
            if spoil:
                g[AT] = big
            e = vb.AdamWTensor.make(tensor(N, pd, 0, 1), g, bits, copy=tensor(N, BF16, 0, 3) if pd == F32 else None, weight_decay=0.1)
            before = e.p.clone()
            opt = vb.AdamW([e])
            opt.step(1, lr=LR, beta1=B1, beta2=B2, eps=EPS, seed=5)
            steps[bits, spoil] = (e, opt)
            if spoil:
                want = (before.cpu()[AT].double() * keep).float().to(pd)
                assert torch.equal(e.p.cpu()[AT], want), bits
                assert e.copy is None or torch.equal(e.copy, e.p.to(BF16))
                rest = torch.ones(N, dtype=torch.bool)
                rest[AT] = False
                assert torch.equal(e.p.cpu()[rest], steps[bits, False][0].p.cpu()[rest])
    e, clean = steps[8, True][0], steps[8, False][0]
    assert torch.isfinite(e.m_scale).all() and torch.isfinite(e.v_scale).all()
    assert torch.isfinite(e.m.float()).all() and torch.isfinite(e.v.float()).all()
    # the block without such a gradient is what it was; 2^63 is within a rounding of the scale of what is held for the others
    assert torch.equal(e.m.view(torch.uint8)[512:768], clean.m.view(torch.uint8)[512:768])
    assert torch.equal(e.v.view(torch.uint8)[512:768], clean.v.view(torch.uint8)[512:768])
    r = (e.v.float() * e.v_scale.repeat_interleave(256)[:N]).cpu().double()
    assert ((r[AT] / 2.0 ** 63 - 1.0).abs() <= 2.0 ** -22).all()
    # and the steps after it, with ordinary gradients, stay finite
    for bits in (32, 8):
        e, opt = steps[bits, True]
        opt.set_grad(0, tensor(N, gd, 0, 7, scale=1e-2))
        for s in (2, 3):
            opt.step(s, lr=LR, beta1=B1, beta2=B2, eps=EPS, seed=5 + s)
        assert torch.isfinite(e.p.float()).all()
        assert e.m.dtype != E4M3 or (torch.isfinite(e.m_scale).all() and torch.isfinite(e.v_scale).all())
