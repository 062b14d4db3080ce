"""A stack with a loss on top and an attention inside: the probe, the status and the checks see these too."""
import numpy as np
import pytest
import torch

from paper_2402_17227_b200 import binding as vb
from tests.test_gpu_train_step import BF16, F32, N, R, T, VOCAB, make, stack_of

pytestmark = pytest.mark.gpu


def exact_grads(st, layers, variants):
    """The layers' dY as the dense pass leaves them (which its own tests hold against the formulas), per variant."""
    out = [[] for _ in layers]
    for v in range(variants):
        st.dense_backward(variant=v)
        for i, L in enumerate(layers):
            out[i].append((L.grad if L.grad is not None else layers[i - 1].dX).clone())
    return out


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_probe_and_ratio_update(dtype):
    """Alg. 1 on layers that were given no gradients: the probe of the exact ones, to the bit; what a backward pass left stays."""
    layers = make(dtype, seed=3, variants=2)
    st = stack_of(layers, dtype)
    grads = exact_grads(st, layers, 2)
    rho, nu = [0.8, 0.7, 0.6], [0.7, 0.6, 0.5]
    want = torch.stack([L.handle.variance_probe(L.X, g, L.W, rho[i], nu[i], 0.9, 40 + i) for i, (L, g) in enumerate(zip(layers, grads))])
    st.backward(rho, nu, seed=4)
    left = [(L.dW.clone(), L.dX.clone(), None if L.grad is None else L.grad.clone(), None if L.norms is None else L.norms.clone())
            for L in layers]
    got = st.probe(rho, nu, 0.9, seed=40)
    assert torch.equal(got, want) and torch.isfinite(got).all() and (got[:, 0] > 0).all()
    for L, before in zip(layers, left):
        for a, b in zip((L.dW, L.dX, L.grad, L.norms), before):
            assert b is None or torch.equal(a, b)
    V = got.cpu().numpy()[::-1]                       # Alg. 1 counts the layers from below
    s, rho2, nu2 = vb.update_ratios(0.9, rho[::-1], nu[::-1], *V.T, layers[0].handle.config)
    assert 0 < s <= 1 and np.all(np.diff(rho2) >= 0) and all(0 < x <= 1 for x in list(rho2) + list(nu2))
    assert st.device_status() == 0
    st.close()


def test_a_layer_that_is_given_its_gradients_is_probed_on_them():
    layers = make(BF16, seed=3, variants=2)
    st = stack_of(layers, BF16)
    grads = exact_grads(st, layers, 2)
    layers[1].dY = [2.0 * g for g in grads[1]]
    got = st.probe([0.5] * 3, [0.5] * 3, 1.0, seed=1)
    for i, L in enumerate(layers):
        g = layers[1].dY if i == 1 else None
        if i == 1:
            assert torch.equal(got[1], L.handle.variance_probe(L.X, g, L.W, 0.5, 0.5, 1.0, 2))
    # the layer below it takes its gradient from that one: twice as large, variances four times
    want = layers[2].handle.variance_probe(layers[2].X, grads[2], layers[2].W, 0.5, 0.5, 1.0, 3)
    assert torch.allclose(got[2, :3], 4.0 * want[:3], rtol=0.05)
    layers[0].loss = None
    with pytest.raises(ValueError):
        st.probe([0.5] * 3, [0.5] * 3, 1.0, seed=1)
    st.close()


def test_status_of_the_loss_and_the_attention_is_the_stacks():
    layers = make(BF16, seed=6)
    st = stack_of(layers, BF16)
    st.backward([1.0] * 3, [1.0] * 3, seed=1)
    assert st.device_status() == 0
    layers[0].loss.tokens[0][5] = VOCAB               # outside the vocabulary
    st.backward([1.0] * 3, [1.0] * 3, seed=1)
    assert st.device_status() == -1 and st.device_status() == 0
    layers[0].loss.tokens[0][5] = 0
    good = layers[2].attention.starts.clone()
    layers[2].attention.starts[N] = R + 1
    st.backward([1.0] * 3, [1.0] * 3, seed=1)
    assert st.device_status() == -1 and st.device_status() == 0
    # both at once are both cleared
    layers[0].loss.tokens[0][5] = VOCAB
    st.backward([1.0] * 3, [1.0] * 3, seed=1)
    assert st.device_status() == -1 and st.device_status() == 0
    layers[2].attention.starts.copy_(good)
    layers[0].loss.tokens[0][5] = 0
    st.backward([1.0] * 3, [1.0] * 3, seed=1)
    assert st.device_status() == 0
    st.close()


@pytest.mark.parametrize("starts", [range(0, R, T), list(range(0, R + 1, T)) + [R], [0, T + 1] + list(range(2 * T, R + 1, T)),
                                    list(range(0, R, T)) + [R - 1]])
def test_starts_that_are_not_those_of_the_data_are_refused(starts):
    layers = make(BF16, seed=6)
    layers[2].attention.starts = torch.tensor(list(starts), dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        stack_of(layers, BF16)
