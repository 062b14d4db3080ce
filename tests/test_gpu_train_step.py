"""A training step through the stack: loss over tokens, its head, an attention between two linears, the optimizer.  Every stage is
checked against its formula in 64 bits on the tensors that it was given, dense and sampled; then the step as a captured graph."""
import numpy as np
import pytest
import torch

from paper_2402_17227_b200 import binding as vb
from paper_2402_17227_b200.stack import AttentionInput, LinearStack, StackLayer, TokenLossInput
from tests.attn_ref import check, reference
from tests.test_gpu_token_loss import backward_of, formulas
from tests.util import rel_fro, tol_for

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
N, T, D, HQ, HK, WIDTH, VOCAB, VOCAB_PAD = 6, 72, 64, 4, 2, 192, 250, 256
R = N * T


def make(dtype, causal=True, seed=0, variants=1):
    """Random weights and one forward pass per variant; layers in backward order: head, attention's output, qkv."""
    g = torch.Generator("cuda").manual_seed(seed)
    randn = lambda *s, k=1.0: (k * torch.randn(*s, generator=g, device="cuda")).to(dtype)
    mul = lambda x, w: (x.float() @ w.float().T).to(dtype)
    w_qkv, w_out, w_head = randn((HQ + 2 * HK) * D, WIDTH, k=0.08), randn(WIDTH, HQ * D, k=0.06), randn(VOCAB_PAD, WIDTH, k=0.2)
    starts = torch.arange(0, R + 1, T, dtype=torch.int32, device="cuda")
    att = AttentionInput(vb.Attention(R, N, HQ, HK, D, dtype, causal=causal), [], [], [], starts)
    loss = TokenLossInput(vb.TokenLoss(R, VOCAB, dtype), [], [], [], [], [], [])
    xs = dict(qkv=[], out=[], head=[])
    for _ in range(variants):
        x = randn(R, WIDTH)
        qkv = mul(x, w_qkv).view(R, HQ + 2 * HK, D)
        o, lse = att.op.fwd(*att.split(qkv), starts)
        att.qkv.append(qkv), att.o.append(o), att.lse.append(lse)
        y = mul(o.view(R, -1), w_out)
        logits = mul(y, w_head)
        xs["qkv"].append(x), xs["out"].append(o.view(R, -1)), xs["head"].append(y)
        tokens = torch.randint(0, VOCAB, (R,), generator=g, device="cuda")
        tokens[torch.rand(R, generator=g, device="cuda") < 0.1] = -1
        # data of different weight, so that the samplers have something to choose from
        weight = torch.exp(torch.randn(N, generator=g, device="cuda")).repeat_interleave(T) / R
        r = loss.op.fwd(logits[:, :VOCAB], tokens)
        loss.logits.append(logits[:, :VOCAB]), loss.tokens.append(tokens), loss.lse.append(r.lse)
        loss.entropy.append(r.entropy), loss.g_logp.append(-weight), loss.g_entropy.append(-0.01 * weight)
    return [StackLayer("head", WIDTH, VOCAB_PAD, w_head, xs["head"], [], loss=loss),
            StackLayer("attn_out", HQ * D, WIDTH, w_out, xs["out"], [], chained=True),
            StackLayer("qkv", WIDTH, (HQ + 2 * HK) * D, w_qkv, xs["qkv"], [], attention=att)]


def stack_of(layers, dtype, **kw):
    return LinearStack(layers, N, T, dtype, **kw)


def np64(t):
    return t.detach().double().cpu().numpy()


def check_pass(layers, dtype, v, sampled):
    """Every layer's gradients from what it was given.  sampled: with the keep probabilities that its handle drew."""
    head, out, qkv = layers
    loss, att = head.loss, qkv.attention
    want, mag, depth = backward_of(loss.logits[v], loss.tokens[v], loss.lse[v], loss.entropy[v], loss.g_logp[v], loss.g_entropy[v])
    u = torch.finfo(dtype).eps / 2
    bound = mag * (2.0 ** -20 + (8 + 3 * depth) * 2.0 ** -24) + 1.01 * u * want.abs() + torch.finfo(dtype).tiny
    assert ((head.grad[:, :VOCAB].double() - want).abs() <= bound).all() and (head.grad[:, VOCAB:] == 0).all()
    sq = head.grad.double().square().sum(1)
    assert torch.allclose(head.norms.double(), sq, rtol=1e-5, atol=1e-37)
    kept_above = None
    for L in layers:
        dY = L.grad if L.grad is not None else head.dX
        alive = np.ones(N, bool)
        if kept_above is not None:
            alive[:] = False
            alive[kept_above] = True
        scale, rows = torch.ones(N, dtype=torch.float64, device="cuda"), torch.ones(R, dtype=torch.float64, device="cuda")
        if sampled:
            s = L.handle.last_sampling()
            g = torch.where(torch.from_numpy(alive).cuda(), dY.double().view(N, -1).nan_to_num(0).norm(dim=1), 0.0)
            assert torch.allclose(s.g.double(), g, rtol=1e-5, atol=1e-30), L.name
            kept = s.idxA.cpu().numpy()
            assert set(kept) <= set(np.flatnonzero(alive)) and np.array_equal(L.kept[:s.cntA].cpu().numpy(), kept)
            scale[:] = 0
            scale[s.idxA.long()] = 1.0 / s.p.double()[s.idxA.long()]
            rows[:] = 0
            rows[s.idxW.long()] = 1.0 / s.q.double()[s.idxW.long()]
            kept_above = kept
        gh = dY.double() * scale.repeat_interleave(T)[:, None]
        gh[scale.repeat_interleave(T) == 0] = 0
        assert rel_fro(np64(L.dW), np64((gh * rows[:, None]).T @ L.X[v].double())) <= tol_for(dtype), L.name
        if L is out:
            # the attention reads this layer's dX; its gradients are those of the kept data
            do = L.dX.double()
            assert rel_fro(np64(do), np64(gh @ L.W.double())) <= tol_for(dtype)
            q, k, vv = att.split(att.qkv[v])
            ref = reference(q, k, vv, att.starts, att.op.causal, D ** -0.5, L.dX.view(R, HQ, D),
                            None if kept_above is None else [int(n) for n in kept_above])
            for name, got in zip(("dq", "dk", "dv"), att.split(qkv.grad.view(R, HQ + 2 * HK, D))):
                check(got, ref[name], what=name)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_dense_and_exact_pass(dtype, causal):
    layers = make(dtype, causal)
    st = stack_of(layers, dtype)
    st.backward([1.0] * 3, [1.0] * 3, seed=1)
    check_pass(layers, dtype, 0, sampled=False)
    exact = [(L.dW.clone(), L.dX.clone()) for L in layers]
    st.dense_backward()
    for L, (dW, dX) in zip(layers, exact):
        assert rel_fro(np64(L.dW), np64(dW)) <= tol_for(dtype)
    assert st.device_status() == 0 and layers[2].attention.op.device_status() == 0 and layers[0].loss.op.device_status() == 0
    st.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kw", [dict(), dict(overlap_layers=True)])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_sampled_pass(dtype, kw, seed):
    layers = make(dtype, seed=seed, variants=2)
    st = stack_of(layers, dtype, **kw)
    for v in (0, 1):
        st.backward([0.8, 0.7, 0.7], [0.7, 0.6, 0.5], seed=seed, variant=v)
        check_pass(layers, dtype, v, sampled=True)
    assert st.device_status() == 0
    st.close()


def test_rows_of_dropped_data_may_stay_unwritten():
    layers = make(BF16, seed=5)
    st = stack_of(layers, BF16)
    st.backward([0.6] * 3, [0.5] * 3, seed=9)
    want = [L.dW.clone() for L in layers]
    st.close()
    layers = make(BF16, seed=5)
    st = stack_of(layers, BF16, skip_dropped_rows=True)
    for L in layers:
        L.dX.fill_(float("nan"))
    layers[2].grad.fill_(float("nan"))
    st.backward([0.6] * 3, [0.5] * 3, seed=9)
    assert all(torch.equal(L.dW, w) for L, w in zip(layers, want))
    st.close()


@pytest.mark.parametrize("dtype,bits", [(F32, 32), (BF16, 32), (BF16, 8)])
def test_captured_step_follows_its_inputs(dtype, bits):
    """Backward and optimizer in one graph; rates and seed on the device.  Three replays are three eager steps, to the bit."""
    runs = []
    for captured in (False, True):
        layers = make(dtype, seed=7)
        st = stack_of(layers, dtype)
        opt = st.make_optimizer(bits, weight_decay=0.01)
        rates, seed = torch.zeros(3, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        whole = lambda: (st.backward([0.7] * 3, [0.6] * 3, seed=4), opt.step(1, lr=0.0, rates=rates, seed_dev=seed))
        set_step = lambda s: (rates.copy_(vb.adamw_rates(1e-3, 0.9, 0.999, s)), seed.fill_(s))
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                whole()
        for s in (1, 2, 3):
            set_step(s)
            if captured:
                graph.replay()
            else:
                whole()
        torch.cuda.synchronize()
        for L, e in zip(layers, opt.tensors):
            if dtype == BF16:
                assert e.copy is L.W and torch.equal(L.W, e.p.to(BF16))
            else:
                assert e.p is L.W
        runs.append([t.clone() for e in opt.tensors for t in (e.p, e.m.view(torch.uint8), e.v.view(torch.uint8))])
        assert st.device_status() == 0
        if captured:
            del graph
        st.close()
    assert all(torch.equal(a, b) for a, b in zip(*runs))
