"""AdamW's table of addresses follows the fields of its tensors."""
import pytest
import torch

from paper_2402_17227_b200 import binding as vb
from tests.test_gpu_adamw import BF16, F32, LR, tensor

pytestmark = pytest.mark.gpu
N = 700


def entry(bits, seed=1):
    return vb.AdamWTensor.make(tensor(N, F32, 0, seed), tensor(N, F32, 0, seed + 1), bits, copy=tensor(N, BF16, 0, seed + 2), weight_decay=0.1)


def states(e):
    return [x.clone() for x in (e.p, e.copy, e.m.view(torch.uint8), e.v.view(torch.uint8))]


NEW = dict(p=lambda: tensor(N, F32, 0, 30), g=lambda: tensor(N, F32, 0, 31), copy=lambda: tensor(N, BF16, 0, 34), weight_decay=lambda: 0.5)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("field", ["p", "g", "bf16 g", "m", "v", "copy", "weight_decay"])
def test_a_field_that_is_set_is_what_the_next_step_uses(bits, field):
    es = [entry(bits, 1), entry(bits, 11)]
    opt, other = vb.AdamW(es), vb.AdamW([es[0]])      # a tensor may be in two lists
    opt.step(1, lr=LR, seed=1)
    e = opt.tensors[0]
    if field in ("m", "v"):
        old = getattr(e, field)
        new = (torch.rand(N, device="cuda") + 0.5).to(old.dtype)
    elif field == "bf16 g":
        new = tensor(N, BF16, 0, 32)
    else:
        new = NEW[field]()
    name = field.split()[-1]
    old = getattr(e, name)
    kept = old.clone() if torch.is_tensor(old) else None
    setattr(e, name, new)
    fresh = vb.AdamWTensor(*[x.clone() if torch.is_tensor(x) else x for x in (e.p, e.g, e.m, e.v, e.m_scale, e.v_scale, e.copy)], e.weight_decay)
    opt.step(2, lr=LR, seed=2)
    vb.AdamW([fresh]).step(2, lr=LR, seed=2)
    assert all(torch.equal(a, b) for a, b in zip(states(e), states(fresh)))
    if kept is not None and name != "weight_decay":   # and the tensor that was there before is left alone
        assert torch.equal(old.view(torch.uint8), kept.view(torch.uint8))
    other.step(3, lr=LR, seed=3)                      # the other list follows too
    vb.AdamW([fresh]).step(3, lr=LR, seed=3)
    assert all(torch.equal(a, b) for a, b in zip(states(e), states(fresh)))


def test_set_grad_beside_other_fields():
    """set_grad after another field has been set must not hide that."""
    a, b = entry(32, 1), entry(32, 1)
    opt = vb.AdamW([a])
    g, p = tensor(N, F32, 0, 40), tensor(N, F32, 0, 41)
    a.p = p.clone()
    opt.set_grad(0, g)
    assert opt.tensors[0].g is g
    b.p, b.g = p.clone(), g
    opt.step(1, lr=LR)
    vb.AdamW([b]).step(1, lr=LR)
    assert all(torch.equal(x, y) for x, y in zip(states(a), states(b)))
    with pytest.raises(ValueError):
        opt.set_grad(0, g[:5])
    assert opt.tensors[0].g is g
    opt.set_grad(0, g.bfloat16())
    b.g = g.bfloat16()
    opt.step(2, lr=LR)
    vb.AdamW([b]).step(2, lr=LR)
    assert all(torch.equal(x, y) for x, y in zip(states(a), states(b)))


def test_a_field_that_does_not_fit_is_refused_by_the_next_step():
    e = entry(32)
    opt = vb.AdamW([e])
    before, g = states(e), e.g
    for bad in (e.g[:5], e.g.double(), e.g.cpu()):
        e.g = bad
        for _ in range(2):
            with pytest.raises(ValueError):
                opt.step(1, lr=LR)
    assert all(torch.equal(x, y) for x, y in zip(before, states(e)))
    e.g = g
    opt.step(1, lr=LR)
    assert not torch.equal(before[0], e.p)
    with pytest.raises(TypeError):
        opt.tensors[0] = e


def test_memory_that_a_tensor_lets_go_of_stays_the_optimizers():
    """`x.data = ...` goes unseen until the field is set: the step meanwhile works on the memory it had, which nobody else has got."""
    e = entry(32)
    opt = vb.AdamW([e])
    was = e.p.data_ptr()
    moved = e.p.clone()
    e.p.data = moved
    others = [torch.zeros(N, device="cuda") for _ in range(8)]
    assert all(x.data_ptr() != was for x in others)
    opt.step(1, lr=LR)
    assert all((x == 0).all() for x in others)
    start = e.p.clone()
    e.p = e.p                                         # follows
    opt.step(2, lr=LR)
    assert not torch.equal(e.p, start)


@pytest.mark.parametrize("name", ["p", "g", "m", "v"])
def test_a_field_that_was_taken_away_is_refused(name):
    e = entry(32)
    opt = vb.AdamW([e])
    old = getattr(e, name)
    setattr(e, name, None)
    with pytest.raises(ValueError):
        opt.step(1, lr=LR)
    with pytest.raises(ValueError):
        opt.set_grad(0, None)
    setattr(e, name, old)
    opt.step(1, lr=LR)
