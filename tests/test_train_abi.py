"""Refusals of the attention, token loss and AdamW entry points that need no GPU: codes, not faults."""
import ctypes as C
import math

import pytest

from paper_2402_17227_b200 import binding as vb
from paper_2402_17227_b200 import build as vbuild


@pytest.fixture(scope="module")
def lib():
    vbuild.build()
    return vb.lib()


def test_null_handles(lib):
    z = C.c_int32(0)
    assert lib.vcas_attn_create(None, None) == lib.vcas_loss_create(None, None) == -1
    assert lib.vcas_attn_destroy(None) == lib.vcas_loss_destroy(None) == -1
    assert lib.vcas_attn_status(None, C.byref(z)) == lib.vcas_loss_status(None, C.byref(z)) == -1
    assert lib.vcas_attn_workspace_bytes(None, None) == lib.vcas_attn_set_wait_limit(None, 1, 0) == -1
    assert lib.vcas_attn_fwd(None, None, None, None, None, 1, 1, None, None, None) == -1
    assert lib.vcas_attn_bwd(None, *[None] * 7, 1, 1, None, None, 0, None, None, None, None) == -1
    assert lib.vcas_loss_fwd(None, None, 0, None, 8, 1, *[None] * 6) == -1
    assert lib.vcas_loss_bwd(None, None, 0, None, 8, 1, *[None] * 5, 0, None, None) == -1


@pytest.mark.parametrize("desc,code", [
    (dict(head_dim=12), -2), (dict(head_dim=0), -2), (dict(head_dim=136), -2), (dict(heads_q=3, heads_kv=2), -2), (dict(heads_kv=0), -2),
    (dict(max_tokens=0), -2), (dict(max_tokens=(1 << 30) + 1), -2), (dict(max_seqs=0), -2), (dict(dtype=2), -3), (dict(scale=-1.0), -1),
    (dict(scale=float("nan")), -1)])
def test_attention_shapes(lib, desc, code):
    d = vb.AttnDesc(**dict(dict(max_tokens=8, max_seqs=2, heads_q=4, heads_kv=2, head_dim=64, dtype=1, causal=0, scale=0.0), **desc))
    h = C.c_void_p(7)
    assert lib.vcas_attn_create(C.byref(h), C.byref(d)) == code and h.value is None


@pytest.mark.parametrize("desc,code", [(dict(max_rows=0), -2), (dict(vocab=0), -2), (dict(top=33), -2), (dict(top=-1), -2),
                                       (dict(vocab=5, top=6), -2), (dict(dtype=9), -3)])
def test_loss_shapes(lib, desc, code):
    d = vb.LossDesc(**dict(dict(max_rows=4, vocab=50, dtype=0, top=2), **desc))
    h = C.c_void_p(7)
    assert lib.vcas_loss_create(C.byref(h), C.byref(d)) == code and h.value is None


def entry(**kw):
    base = dict(p=64, g=64, m=64, v=64, m_scale=None, v_scale=None, copy=None, n=8, weight_decay=0.0, p_dtype=0, g_dtype=0, state_bits=32)
    return vb.AdamWEntry(**dict(base, **kw))


@pytest.mark.parametrize("kw,code", [
    (dict(p=None), -1), (dict(g=None), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(n=-1), -2), (dict(n=(1 << 34) + 1), -2),
    (dict(state_bits=16), -3), (dict(p_dtype=3), -3), (dict(g_dtype=-1), -3), (dict(state_bits=8), -1), (dict(weight_decay=-1.0), -1),
    (dict(weight_decay=float("inf")), -1), (dict(p_dtype=1, copy=64), -3), (dict(p=65), -1), (dict(g=66), -1), (dict(m=67), -1)])
def test_adamw_tensors(lib, kw, code):
    a = vb.AdamWArgs(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    e = (vb.AdamWEntry * 1)(entry(**kw))
    assert lib.vcas_adamw_step(e, 1, C.byref(a), None) == code


@pytest.mark.parametrize("kw", [dict(step=0), dict(beta1=1.0), dict(beta2=1.5), dict(lr=-1.0), dict(lr=float("nan")), dict(eps=float("inf"))])
def test_adamw_rates_refused(lib, kw):
    a = vb.AdamWArgs(**dict(dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1), **kw))
    assert lib.vcas_adamw_step(None, 0, C.byref(a), None) == -1
    assert lib.vcas_adamw_step(None, 1, C.byref(a), None) == -1 and lib.vcas_adamw_step(None, -1, C.byref(a), None) == -1


def test_adamw_without_tensors_and_rates(lib):
    a = vb.AdamWArgs(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    assert lib.vcas_adamw_step(None, 0, C.byref(a), None) == 0
    assert lib.vcas_adamw_step((vb.AdamWEntry * 1)(entry(n=0, p=None)), 1, C.byref(a), None) == 0      # nothing to launch
    r = vb.adamw_rates(1e-3, 0.9, 0.999, 7).double()
    want = (1e-3, 1e-3 / (1 - 0.9 ** 7), 1 / math.sqrt(1 - 0.999 ** 7))
    assert all(abs(float(x) - w) <= 2.0 ** -24 * w for x, w in zip(r, want))
