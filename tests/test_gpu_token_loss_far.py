"""Gradient of rows whose logits lie far from 0: p is the softmax of the logits, not what an lse rounded to fp32 leaves of it."""
import pytest
import torch

from paper_2402_17227_b200 import binding as vb
from tests.test_gpu_token_loss import BF16, F, F32, close, formulas, logits_of, tokens_of

pytestmark = pytest.mark.gpu


def far_rows(rows, vocab, dtype, pad, off):
    """Rows at the type's lowest value (throughout, but for a few values, with -inf between), around +-2000, +-30000 and +-1e30, on a
    grid that the type holds, and ordinary ones."""
    x = logits_of(rows, vocab, dtype, pad, off, seed=3)
    lowest = torch.finfo(dtype).min
    g = torch.Generator("cuda").manual_seed(4)
    steps = torch.randint(-4, 5, (rows, vocab), generator=g, device="cuda").float()
    for r in range(rows):
        kind = r % 10
        if kind in (0, 1, 2):
            x[r] = lowest
        if kind == 1:
            x[r, vocab // 2:vocab // 2 + 3] = torch.finfo(dtype).min / 2
        if kind == 2:
            x[r, ::2] = float("-inf")
        if kind in (3, 4, 5, 6):
            size = (2000.0, -2000.0, 30000.0, -30000.0)[kind - 3]
            grain = 2.0 if dtype == F32 else max(1.0, abs(size) / 128)        # a few steps of the type
            x[r] = (size + grain * steps[r]).to(dtype)
        if kind in (7, 8):
            x[r] = torch.where(steps[r] > 2, 1e30, -1e30).to(dtype) * (1 if kind == 7 else -1)
    return x


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab,pad,off", [(1, 0, 0), (3, 2, 1), (50, 0, 3), (1000, 0, 0), (4099, 5, 7), (32000, 0, 0)])
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("rows", [10, 640])
def test_gradient_of_rows_far_from_zero(dtype, vocab, pad, off, entropy, rows):
    x = far_rows(rows, vocab, dtype, pad, off)
    tokens = tokens_of(rows, vocab)
    op = vb.TokenLoss(rows, vocab, dtype)
    r = op.fwd(x, tokens)
    lse, _, H, _, _, lp, p = formulas(x, tokens, 1)
    g = torch.Generator("cuda").manual_seed(8)
    gl = torch.randn(rows, generator=g, device="cuda")
    ge = torch.randn(rows, generator=g, device="cuda") if entropy else None
    kw = dict(entropy=H.float(), g_entropy=ge) if entropy else {}
    has = torch.where((tokens >= 0) & (lse != float("-inf")), gl.double(), 0.0)[:, None]        # no distribution, no gradient
    onehot = torch.zeros_like(p).scatter_(1, tokens.clamp_min(0)[:, None], 1.0)
    want, mag = has * (onehot - p), has.abs() * (onehot + p)
    depth = torch.where(p > 0, lp.abs(), 0.0)
    Hd = H.float().double()[:, None]
    if entropy:
        want = want - torch.where(p > 0, ge.double()[:, None] * p * (lp + Hd), 0.0)
        mag = mag + torch.where(p > 0, ge.double().abs()[:, None] * p * (depth + Hd.abs()), 0.0)
    # log p is off by half a step of lse (2^-15) below 1024, above that by the logarithm's ulp (2^-20 up to 16), an exponential's error in the sum
    # (2^-21, 3 F d of its argument) and the sum's additions (vocab / threads, at most vocab / 32: F each); then as anywhere: exp 2^-21, its argument 3 F |log p|,
    # five fp32 operations, the stored value's rounding.  An exponential below 2^-126 is 0.
    ge_abs = ge.double().abs()[:, None] if entropy else 0.0
    far = 2.0 ** -19 + (vocab / 32 + 8) * F + 3 * F * (p * depth).sum(1)
    slack = torch.where(lse.abs() < 1024, 2.0 ** -15, far)[:, None] + 2.0 ** -20 + (8 + 3 * depth) * F
    lost = 2.0 ** -126 * (has.abs() + ge_abs * (depth + Hd.abs()))
    bound = slack * (mag + ge_abs * p) + lost + 1.01 * torch.finfo(dtype).eps / 2 * want.abs() + torch.finfo(dtype).tiny
    for out in (None, logits_of(rows, vocab, dtype, pad + 1, off, seed=9)):
        d, norms = op.bwd(x, tokens, r.lse, gl, dlogits=out, **kw)
        close(d, want, bound, "dlogits")
        sq = d.double().square().sum(1)
        close(norms, sq, sq * (vocab / 32 + 16) * F + 1e-37, "row norms")
    same = x.clone()
    assert torch.equal(op.bwd(same, tokens, r.lse, gl, dlogits=same, **kw)[0], d)
    assert op.device_status() == 0
