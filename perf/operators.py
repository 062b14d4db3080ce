"""What a training step does before and behind the sampled backward of its linear layers, as cases that can be timed.

Three operators: attention over packed sequences (forward, and backward over the data that SampleA kept), the log
probabilities of given tokens (with entropy and top alternatives, and the gradient that starts the backward pass), and
an AdamW step over many tensors (states in 32 bits, or in 8 with a scale for each block of 256).  `run` computes them in
plain torch operations, or, with `own`, through this framework.  `listed` names twelve calls; `draw` gives others.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 256                      # elements under one scale of an 8-bit state


def _binding():
    from paper_2402_17227_b200 import binding
    return binding


def _attn(name, kind, dtype, N, T, heads, kv_heads, dim, causal, ragged, fused, kept=1.0):
    """kind: attn_fwd | attn_bwd.  N sequences of T tokens (ragged: of one to T, drawn by N and T).  fused: q, k and v lie in
    one buffer, as the projection leaves them.  kept: share of the sequences whose gradient is not zero."""
    return dict(name=name, kind=kind, dtype=dtype, N=N, T=T, heads=heads, kv_heads=kv_heads, dim=dim, causal=causal,
                ragged=ragged, fused=fused, kept=kept)


def _loss(name, kind, dtype, rows, vocab, pad, top, ignored, banned, entropy):
    """kind: loss_fwd | loss_bwd.  pad: unused columns behind each row.  ignored: share of rows without a token.  banned:
    share of the vocabulary at -inf.  entropy: the loss has an entropy term (backward)."""
    return dict(name=name, kind=kind, dtype=dtype, rows=rows, vocab=vocab, pad=pad, top=top, ignored=ignored, banned=banned,
                entropy=entropy)


def _adamw(name, bits, grad, width, ff, blocks, copy, odd):
    """Tensors of `blocks` transformer blocks (four matrices, their biases, two norms).  copy: a bf16 copy of the weights is
    written too.  odd: elements that the first tensor has beyond its matrix."""
    return dict(name=name, kind="adamw", bits=bits, grad=grad, width=width, ff=ff, blocks=blocks, copy=copy, odd=odd)


def listed():
    return [
        # the smallest layer in use, four sequences of 64 tokens in full precision: launches and latency
        _attn("attn_fwd_fp32_small", "attn_fwd", "fp32", 4, 64, 4, 4, 64, False, False, False),
        # fine-tuning a base-sized encoder on sentences of different lengths, nothing padded
        _attn("attn_fwd_base_packed", "attn_fwd", "bf16", 32, 128, 12, 12, 64, False, True, True),
        # the backward of a vision transformer's attention, 197 tokens, on the data that SampleA kept
        _attn("attn_bwd_vit_kept", "attn_bwd", "bf16", 64, 197, 12, 12, 64, False, False, True, 0.4),
        # a decoder's prompt: causal, grouped heads
        _attn("attn_fwd_llm", "attn_fwd", "bf16", 8, 2048, 32, 8, 128, True, False, True),
        # its backward over packed sequences of one to 2048 tokens
        _attn("attn_bwd_llm_packed", "attn_bwd", "bf16", 16, 2048, 32, 8, 128, True, True, True),
        # scores of a few sampled tokens: few rows, twenty alternatives, half of the vocabulary not allowed
        _loss("loss_fwd_few_rows", "loss_fwd", "bf16", 8, 32000, 0, 20, 0.0, 0.5, False),
        # a policy's log probabilities and entropy over a large vocabulary
        _loss("loss_fwd_large_vocab", "loss_fwd", "bf16", 4096, 131072, 0, 5, 0.1, 0.0, False),
        # the gradient of a masked language model's loss: odd vocabulary, padded rows, most positions without a token
        _loss("loss_bwd_mlm_fp32", "loss_bwd", "fp32", 4096, 30522, 6, 0, 0.85, 0.0, False),
        # the gradient of a decoder's loss with an entropy term
        _loss("loss_bwd_llm", "loss_bwd", "bf16", 16384, 32000, 0, 0, 0.05, 0.0, True),
        # one small layer's tensors: latency
        _adamw("adamw_small", 32, "fp32", 256, 256, 1, True, 1),
        # eight blocks of a large encoder, gradients as the sampled backward leaves them (fp32)
        _adamw("adamw_bert_large", 32, "fp32", 1024, 4096, 8, True, 0),
        # two blocks of an LLM with 8-bit states and bf16 gradients
        _adamw("adamw_llm_8bit", 8, "bf16", 4096, 11008, 2, True, 0),
    ]


def _log_int(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over its logarithm."""
    v = lo * (hi / lo) ** rng.random()
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["attn_fwd", "attn_bwd", "loss_fwd", "loss_bwd", "adamw"])
    if kind.startswith("attn"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        dim = rng.choice([64, 64, 128, 128, _log_int(rng, 16, 128, 8)])
        groups = rng.choice([1, 1, 2, 4, 8])
        heads = groups * _log_int(rng, 1, 32 // groups)
        T = _log_int(rng, 1, 2048 if dtype == "bf16" else 512)
        N = _log_int(rng, 1, max(1, min(64, (16384 if dtype == "bf16" else 4096) // T)))
        c = _attn("", kind, dtype, N, T, heads, heads // groups, dim, rng.random() < 0.5, rng.random() < 0.5,
                  rng.random() < 0.5, rng.choice([1.0, 1.0, 0.5]) if kind == "attn_bwd" else 1.0)
    elif kind.startswith("loss"):
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        vocab = _log_int(rng, 50, 131072)
        rows = _log_int(rng, 1, max(1, min(16384, (1 << 28) // vocab)))
        c = _loss("", kind, dtype, rows, vocab, rng.choice([0, 0, 1, 6, 64]), rng.choice([0, 1, 5, 20]) if kind == "loss_fwd" else 0,
                  rng.choice([0.0, 0.1, 0.85]), rng.choice([0.0, 0.0, 0.5]), kind == "loss_bwd" and rng.random() < 0.5)
    else:
        width = _log_int(rng, 8, 4096)
        c = _adamw("", rng.choice([8, 32]), rng.choice(["fp32", "bf16"]), width, _log_int(rng, width, 3 * width),
                   _log_int(rng, 1, max(1, min(24, (1 << 24) // (width * width)))), rng.random() < 0.5, _log_int(rng, 1, 999))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ sizes
def _lengths(c):
    if not c["ragged"]:
        return [c["T"]] * c["N"]
    rng = random.Random(c["N"] * 65537 + c["T"])
    lens = [_log_int(rng, max(1, c["T"] // 16), c["T"]) for _ in range(c["N"])]
    lens[rng.randrange(c["N"])] = c["T"]
    if c["N"] > 2:
        lens[0], lens[-1] = 1, 0 if c["T"] == 1 else lens[-1]
    return lens


def _kept(c):
    rng = random.Random(c["N"] * 31 + c["T"])
    n = max(1, round(c["N"] * c["kept"]))
    return sorted(rng.sample(range(c["N"]), n))


def _sizes(c):
    """Elements of every tensor of an optimizer step, and whether it decays."""
    d, ff = c["width"], c["ff"]
    block = [(d * 3 * d, True), (3 * d, False), (d * d, True), (d, False), (d * ff, True), (ff, False), (ff * d, True), (d, False)]
    block += [(d, False)] * 4
    sizes = block * c["blocks"]
    return [(sizes[0][0] + c["odd"], True)] + sizes[1:]


def _arena(c):
    """Sizes, offsets (each tensor starts on a block) and total length of the flat buffers that hold all tensors."""
    sizes = _sizes(c)
    off, at = [], 0
    for n, _ in sizes:
        off.append(at)
        at += (n + BLOCK - 1) // BLOCK * BLOCK
    return sizes, off, at


# ----------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    return dev, torch.Generator(dev).manual_seed(seed % (1 << 31) + 1)


def _prepare_attn(c, seed):
    dev, g = _generator(seed)
    dt, D, Hq, Hk = DTYPES[c["dtype"]], c["dim"], c["heads"], c["kv_heads"]
    lens = _lengths(c)
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    total = starts[-1]
    s = dict(kind=c["kind"], case=c, dtype=dt, starts=torch.tensor(starts, dtype=torch.int32, device=dev), T=max(lens),
             lens=torch.tensor(lens, device=dev))
    randn = lambda *shape: torch.randn(*shape, generator=g, device=dev).to(dt)  # noqa: E731
    if c["fused"]:
        qkv = randn(total, Hq + 2 * Hk, D)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    else:
        s["q"], s["k"], s["v"] = randn(total, Hq, D), randn(total, Hk, D), randn(total, Hk, D)
    if c["kind"] == "attn_bwd":
        s["o"], s["lse"] = _plain_attention(s)
        s["do"] = randn(total, Hq, D)
        kept = _kept(c)
        s["alive"] = torch.zeros(c["N"], dtype=torch.int32, device=dev)
        s["alive"][:len(kept)] = torch.tensor(kept, dtype=torch.int32, device=dev)
        s["alive_cnt"] = torch.tensor([len(kept)], dtype=torch.int32, device=dev)
        if c["fused"]:
            dqkv = torch.zeros(total, Hq + 2 * Hk, D, dtype=dt, device=dev)
            s["dq"], s["dk"], s["dv"] = dqkv[:, :Hq], dqkv[:, Hq:Hq + Hk], dqkv[:, Hq + Hk:]
        else:
            s["dq"], s["dk"], s["dv"] = (torch.zeros(total, h, D, dtype=dt, device=dev) for h in (Hq, Hk, Hk))
    else:
        s["o"] = torch.zeros(total, Hq, D, dtype=dt, device=dev)
        s["lse"] = torch.zeros(Hq, total, dtype=torch.float32, device=dev)
    if own:
        s["op"] = _binding().Attention(total, c["N"], Hq, Hk, D, dt, causal=c["causal"])
    return s


def _prepare_loss(c, seed):
    dev, g = _generator(seed)
    R, V, dt = c["rows"], c["vocab"], DTYPES[c["dtype"]]
    store = torch.full((R, V + c["pad"]), float("nan"), dtype=dt, device=dev)
    logits = store[:, :V]
    step = max(1, (1 << 27) // V)            # rows at a time, so that the draws in fp32 stay small
    tokens = torch.randint(0, V, (R,), generator=g, device=dev)
    for r in range(0, R, step):
        x = 2.5 * torch.randn(min(step, R - r), V, generator=g, device=dev)
        # a model that has learned something: the given token stands out
        x.scatter_add_(1, tokens[r:r + step, None], 8.0 * torch.rand(x.shape[0], 1, generator=g, device=dev))
        logits[r:r + step] = x.to(dt)
    if c["banned"] > 0:
        ban = torch.rand(V, generator=g, device=dev) < c["banned"]
        ban[:32] = False
        logits.masked_fill_(ban[None], float("-inf"))
    tokens[torch.rand(R, generator=g, device=dev) < c["ignored"]] = -1
    s = dict(kind=c["kind"], case=c, logits=logits, tokens=tokens)
    if c["kind"] == "loss_bwd":
        got = _plain_loss(s, 0)
        s["lse"], s["entropy"] = got["lse"], got["entropy"]
        s["g_logp"] = -torch.rand(R, generator=g, device=dev) / R
        s["g_entropy"] = torch.full((R,), -0.01 / R, device=dev) if c["entropy"] else None
        s["dlogits"] = torch.zeros(R, V + c["pad"], dtype=dt, device=dev)[:, :V]
        s["norms"] = torch.zeros(R, dtype=torch.float32, device=dev)
    if own:
        s["op"] = _binding().TokenLoss(R, V, dt, top=c["top"])
    return s


def _prepare_adamw(c, seed):
    dev, g = _generator(seed)
    sizes, off, total = _arena(c)
    nblk = total // BLOCK
    s = dict(kind="adamw", case=c, seed=seed % 65521, sizes=sizes, off=off)
    inside = torch.zeros(total + 1, dtype=torch.int8, device=dev)         # 1 on elements of a tensor, 0 behind its end
    inside[torch.tensor(off, device=dev)] += 1
    inside[torch.tensor([o + n for o, (n, _) in zip(off, sizes)], device=dev)] -= 1
    inside = inside.cumsum(0, dtype=torch.int8)[:total]
    s["p"] = 0.02 * torch.randn(total, generator=g, device=dev) * inside
    size = torch.exp(1.5 * torch.randn(nblk, 1, generator=g, device=dev)) * 1e-3      # gradients differ from layer to layer
    s["g"] = ((torch.randn(nblk, BLOCK, generator=g, device=dev) * size).view(-1) * inside).to(DTYPES[c["grad"]])
    if c["bits"] == 32:
        s["m"] = (0.3 * torch.randn(nblk, BLOCK, generator=g, device=dev) * size).view(-1) * inside
        s["v"] = ((0.3 + torch.rand(nblk, BLOCK, generator=g, device=dev)) * size).square().view(-1) * inside
    else:
        m = torch.randn(nblk, BLOCK, generator=g, device=dev).clamp_(-4, 4) * inside.view(nblk, BLOCK)
        r = (0.3 + torch.rand(nblk, BLOCK, generator=g, device=dev)) * inside.view(nblk, BLOCK)
        scale = lambda x: (448.0 / x.abs().amax(1, keepdim=True).clamp_min(1e-30))  # noqa: E731
        s["m"] = (m * scale(m)).clamp_(-448, 448).to(torch.float8_e4m3fn).view(-1)
        s["v"] = (r * scale(r)).clamp_(-448, 448).to(torch.float8_e4m3fn).view(-1)
        s["m_scale"] = (size * (1.0 / 448.0)).view(-1).contiguous()
        s["v_scale"] = (size * (1.3 / 448.0)).view(-1).contiguous()
    if c["copy"]:
        s["copy"] = torch.zeros(total, dtype=torch.bfloat16, device=dev)
    s["hyper"] = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=100)
    s["decay"] = [0.01 if d else 0.0 for _, d in sizes]
    if own:
        vb = _binding()
        part = lambda x, o, n, b=1: x[o // b:o // b + (n + b - 1) // b] if x is not None else None  # noqa: E731
        s["op"] = vb.AdamW([vb.AdamWTensor(part(s["p"], o, n), part(s["g"], o, n), part(s["m"], o, n), part(s["v"], o, n),
                                           m_scale=part(s.get("m_scale"), o, n, BLOCK), v_scale=part(s.get("v_scale"), o, n, BLOCK),
                                           copy=part(s.get("copy"), o, n), weight_decay=d)
                            for (n, _), o, d in zip(sizes, off, s["decay"])])
    return s


def prepare(case, seed):
    """Inputs, outputs and states that a training program holds, and its handles."""
    if case["kind"].startswith("attn"):
        return _prepare_attn(case, seed)
    return _prepare_loss(case, seed) if case["kind"].startswith("loss") else _prepare_adamw(case, seed)


# ------------------------------------------------------------------------------------------- plain forms
def _padded(s, x, heads):
    """[total, h, D] -> [N, heads, T, D] in fp32, zeros behind each sequence, shared heads repeated."""
    at, ok = _places(s)
    y = torch.where(ok[:, :, None, None], x.float()[at], 0.0)
    return y.permute(0, 2, 1, 3).repeat_interleave(heads // x.shape[1], 1)


def _places(s):
    t = torch.arange(s["T"], device=s["q"].device)
    ok = t < s["lens"][:, None]
    return torch.where(ok, s["starts"][:-1, None].long() + t, 0), ok


def _packed(s, y):
    """[N, h, T, D] -> [total, h, D] in the layer's type."""
    return y.permute(0, 2, 1, 3)[_places(s)[1]].to(s["dtype"])


def _scores(s):
    """Scaled scores [N, Hq, T, T] with -inf where a row does not look."""
    c = s["case"]
    q, k = _padded(s, s["q"], c["heads"]), _padded(s, s["k"], c["heads"])
    x = q @ k.transpose(-1, -2)
    x *= 1.0 / math.sqrt(c["dim"])
    t = torch.arange(s["T"], device=x.device)
    see = t < s["lens"][:, None, None, None]
    if c["causal"]:
        see = see & (t <= t[:, None])
    return x.masked_fill_(~see, float("-inf")), q, k


def _plain_attention(s):
    x, _, _ = _scores(s)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x @ _padded(s, s["v"], s["case"]["heads"])) / total
    lse = (top + total.log())[..., 0]
    return _packed(s, o), lse.transpose(1, 2)[_places(s)[1]].t().contiguous()


def _plain_attention_bwd(s):
    c = s["case"]
    x, q, k = _scores(s)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    p = p.div_(p.sum(-1, keepdim=True).clamp_min_(1e-30))
    alive = torch.zeros(c["N"], device=p.device).index_fill_(0, s["alive"][:len(_kept(c))].long(), 1.0)
    do = _padded(s, s["do"], c["heads"]) * alive[:, None, None, None]
    v = _padded(s, s["v"], c["heads"])
    by_group = lambda y: y.unflatten(1, (c["kv_heads"], -1)).sum(2)  # noqa: E731
    dv = by_group(p.transpose(-1, -2) @ do)
    dp = do @ v.transpose(-1, -2)
    dp -= (dp * p).sum(-1, keepdim=True)
    ds = p.mul_(dp).mul_(1.0 / math.sqrt(c["dim"]))
    return [_packed(s, ds @ k), _packed(s, by_group(ds.transpose(-1, -2) @ q)), _packed(s, dv)]


def _plain_loss(s, k):
    x = s["logits"].float()
    tokens = s["tokens"]
    top = x.amax(1, keepdim=True)
    e = (x - top).exp_()
    total = e.sum(1, keepdim=True)
    lse = top + total.log()
    # entropy = log sum - sum p (x - max), with 0 for p = 0
    e *= torch.where(x == float("-inf"), 0.0, x - top)
    out = dict(lse=lse[:, 0], entropy=(total.log() - e.sum(1, keepdim=True) / total)[:, 0])
    given = x.gather(1, tokens.clamp_min(0)[:, None])[:, 0] - lse[:, 0]
    out["logp"] = torch.where(tokens < 0, 0.0, given)
    if k:
        # larger values first, then lower indices: both in one 64-bit key
        bits = (x + 0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = (key << 32) | (0x7FFFFFFF - torch.arange(x.shape[1], device=x.device))
        ids = 0x7FFFFFFF - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)
        out["top_ids"] = ids.int()
        out["top_logp"] = x.gather(1, ids) - lse
    return out


def _plain_loss_bwd(s):
    x = s["logits"].float()
    lp = x - s["lse"][:, None]
    p = lp.exp()
    gl = torch.where(s["tokens"] < 0, 0.0, s["g_logp"])[:, None]
    d = -gl * p
    if s["g_entropy"] is not None:
        d -= s["g_entropy"][:, None] * p * torch.where(p == 0, 0.0, lp + s["entropy"][:, None])
    d.scatter_add_(1, s["tokens"].clamp_min(0)[:, None], gl)
    d = d.to(s["logits"].dtype)
    return [d, d.float().square().sum(1)]


def _philox_bytes(s, total, device):
    """Eight random bits for the first state and eight for the second, of every element: word e // 2 of the Philox4x32-10 output
    of counter (element // 8 within the tensor, tensor, 3, 0) holds those of elements e and e + 1 of the eight."""
    n = torch.tensor([(n + BLOCK - 1) // BLOCK * (BLOCK // 8) for n, _ in s["sizes"]], device=device)
    c1 = torch.repeat_interleave(torch.arange(len(n), device=device), n)
    c0 = torch.arange(total // 8, device=device) - torch.repeat_interleave(n.cumsum(0) - n, n)
    c2, c3 = torch.full_like(c0, 3), torch.zeros_like(c0)
    k0, k1, mask = s["seed"], 0, 0xFFFFFFFF
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & mask) ^ c1 ^ k0, b & mask, ((a >> 32) & mask) ^ c3 ^ k1, a & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    w = torch.stack([c0, c1, c2, c3], 1)[:, :, None] >> torch.tensor([0, 16], device=device)
    w = w.view(-1)                            # per element: bits 0-7 for the first state, 8-15 for the second
    return (w & 255).int(), ((w >> 8) & 255).int()


def _to_8bit(x, rnd, least):
    """x in blocks -> (e4m3 values, scale a block): scale = largest / 448; x / scale goes up or down to a neighbouring value, by
    where it lies between them and the random bits.  least: 1 where a positive x must not become 0."""
    big = x.abs().amax(1, keepdim=True)
    scale = big * (1.0 / 448.0)
    y = torch.where(big > 0, x.abs() * (448.0 / big), 0.0).clamp_max_(448.0)
    bits = (y * 2.0 ** -120).view(torch.int32)                 # its exponent and mantissa now end at bit 20
    code = (bits + (rnd.view_as(bits) << 12) + 2048) >> 20
    code = torch.where(x > 0, code.clamp_min(least), code)
    code = (code | ((x < 0).int() << 7)).to(torch.uint8)
    return code.view(torch.float8_e4m3fn), scale


def _plain_adamw(s):
    c, h = s["case"], s["hyper"]
    b1, b2 = h["beta1"], h["beta2"]
    f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
    step_size = f32(h["lr"] / (1.0 - b1 ** h["step"]))
    inv = f32(1.0 / math.sqrt(1.0 - b2 ** h["step"]))
    dev, total = s["p"].device, s["p"].numel()
    n = torch.tensor([(n + BLOCK - 1) // BLOCK * BLOCK for n, _ in s["sizes"]], device=dev)
    keep = torch.repeat_interleave(torch.tensor([1.0 - h["lr"] * d for d in s["decay"]], device=dev), n)
    g = s["g"].float()
    if c["bits"] == 32:
        s["m"].mul_(f32(b1)).add_(g * f32(1.0 - b1))
        s["v"].mul_(f32(b2)).add_(g * g * f32(1.0 - b2))
        m, root = s["m"], s["v"].sqrt()
    else:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1) * f32(b1) + g * f32(1.0 - b1)
        r = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
        root = (r * r * f32(b2) + g * g * f32(1.0 - b2)).sqrt()
        r1, r2 = _philox_bytes(s, total, dev)
        for name, value, rnd, least in (("m", m, r1, 0), ("v", root, r2, 1)):
            code, scale = _to_8bit(value.view(-1, BLOCK), rnd, least)
            s[name].copy_(code.view(-1))
            s[name + "_scale"].copy_(scale[:, 0])
    s["p"].mul_(keep).sub_(m * step_size / (root * inv + f32(h["eps"])))
    if c["copy"]:
        s["copy"].copy_(s["p"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return {k: s[k] for k in ("p", "copy", "m", "v", "m_scale", "v_scale") if k in s}


def run(s):
    kind = s["kind"]
    if kind == "attn_fwd":
        if own:
            return list(s["op"].fwd(s["q"], s["k"], s["v"], s["starts"], o=s["o"], lse=s["lse"]))
        return list(_plain_attention(s))
    if kind == "attn_bwd":
        if own:
            return list(s["op"].bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["starts"], dq=s["dq"], dk=s["dk"],
                                    dv=s["dv"], alive_in=s["alive"], alive_cnt_in=s["alive_cnt"]))
        return _plain_attention_bwd(s)
    if kind == "loss_fwd":
        if own:
            r = s["op"].fwd(s["logits"], s["tokens"])
            out = dict(lse=r.lse, entropy=r.entropy, logp=r.logp)
            return dict(out, top_ids=r.top_ids, top_logp=r.top_logp) if s["case"]["top"] else out
        return _plain_loss(s, s["case"]["top"])
    if kind == "loss_bwd":
        if own:
            return list(s["op"].bwd(s["logits"], s["tokens"], s["lse"], s["g_logp"], entropy=s["entropy"],
                                    g_entropy=s["g_entropy"], dlogits=s["dlogits"], a_out=s["norms"]))
        return _plain_loss_bwd(s)
    if own:
        h = s["hyper"]
        s["op"].step(h["step"], lr=h["lr"], beta1=h["beta1"], beta2=h["beta2"], eps=h["eps"], seed=s["seed"])
        return _adamw_outputs(s)
    return _plain_adamw(s)


# ------------------------------------------------------------------------------------------------- work
def work(case):
    c = case
    if c["kind"].startswith("attn"):
        lens = _lengths(c)
        b = 4 if c["dtype"] == "fp32" else 2
        bwd = c["kind"] == "attn_bwd"
        seen = [lens[i] for i in _kept(c)] if bwd else lens
        pairs = sum(n * (n + 1) // 2 if c["causal"] else n * n for n in seen)
        row = c["dim"] * b
        q, kv, tokens = row * c["heads"], row * c["kv_heads"], sum(seen)
        if bwd:      # q, o, do, k, v and lse of the kept data; the gradients of all
            by = tokens * (3 * q + 2 * kv + 4 * c["heads"]) + sum(lens) * (q + 2 * kv)
        else:
            by = tokens * (2 * q + 2 * kv + 4 * c["heads"])
        return {"bytes": float(by), "flops": float((10 if bwd else 4) * c["dim"] * c["heads"] * pairs)}
    if c["kind"].startswith("loss"):
        n, b = c["rows"] * c["vocab"], 4 if c["dtype"] == "fp32" else 2
        if c["kind"] == "loss_bwd":
            return {"bytes": float(2 * n * b + c["rows"] * 28), "flops": 6.0 * n}
        return {"bytes": float(n * b + c["rows"] * (20 + 8 * c["top"])), "flops": 6.0 * n}
    n = sum(x for x, _ in _sizes(c))
    each = 8 + (4 if c["grad"] == "fp32" else 2) + (2 if c["copy"] else 0) + (16 if c["bits"] == 32 else 4 + 16 / BLOCK)
    return {"bytes": float(n * each), "flops": 15.0 * n}


# ------------------------------------------------------------------------------- the definition in 64 bits
def _exact_attention(c, s):
    """Sequence by sequence and head by head, as the formulas stand."""
    starts = s["starts"].tolist()
    group = c["heads"] // c["kv_heads"]
    bwd = c["kind"] == "attn_bwd"
    kept = set(_kept(c))
    q, k, v = (s[n].double() for n in "qkv")
    o, lse = torch.zeros_like(q), torch.zeros(c["heads"], q.shape[0], dtype=torch.float64, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for n in range(c["N"]):
        t = slice(starts[n], starts[n + 1])
        L = starts[n + 1] - starts[n]
        if L == 0 or (bwd and n not in kept):
            continue
        for h in range(c["heads"]):
            K, V = k[t, h // group], v[t, h // group]
            S = torch.einsum("id,jd->ij", q[t, h], K) / c["dim"] ** 0.5
            if c["causal"]:
                S = S + torch.full((L, L), float("-inf"), dtype=torch.float64, device=S.device).triu(1)
            l = torch.logsumexp(S, 1)
            P = torch.exp(S - l[:, None])
            if not bwd:
                o[t, h], lse[h, t] = P @ V, l
                continue
            dO = s["do"][t, h].double()
            dP = torch.einsum("id,jd->ij", dO, V)
            dS = P * (dP - torch.einsum("ij,ij->i", P, dP)[:, None]) / c["dim"] ** 0.5
            dq[t, h] = torch.einsum("ij,jd->id", dS, K)
            dk[t, h // group] += torch.einsum("ij,id->jd", dS, q[t, h])
            dv[t, h // group] += torch.einsum("ij,id->jd", P, dO)
    return [dq, dk, dv] if bwd else [o, lse]


def _exact_loss(c, s):
    parts = []
    R, V = s["logits"].shape
    step = max(1, (1 << 25) // V)
    for r in range(0, R, step):
        x, tok = s["logits"][r:r + step].double(), s["tokens"][r:r + step]
        lp = torch.log_softmax(x, 1)
        p = lp.exp()
        plp = torch.where(p > 0, p * lp, 0.0)
        rows, has = torch.arange(len(tok), device=tok.device), tok >= 0
        H = -plp.sum(1)
        if c["kind"] == "loss_fwd":
            one = dict(lse=torch.logsumexp(x, 1), entropy=H, logp=torch.where(has, lp[rows, tok.clamp_min(0)], 0.0))
            if c["top"]:
                val, ids = torch.sort(x, dim=1, descending=True, stable=True)
                one["top_ids"] = ids[:, :c["top"]].int()
                one["top_logp"] = lp.gather(1, ids[:, :c["top"]])
        else:
            onehot = torch.zeros_like(p)
            onehot[rows[has], tok[has]] = 1.0
            d = torch.where(has, s["g_logp"][r:r + step].double(), 0.0)[:, None] * (onehot - p)
            if s["g_entropy"] is not None:
                d = d - s["g_entropy"][r:r + step, None].double() * (plp + p * H[:, None])
            one = dict(d=d.to(s["logits"].dtype) if V * R > (1 << 29) else d, norm=d.to(s["logits"].dtype).double().square().sum(1))
        parts.append(one)
    cat = {k: torch.cat([x[k] for x in parts]) for k in parts[0]}
    return [cat["d"], cat["norm"]] if c["kind"] == "loss_bwd" else cat


def _exact_adamw(c, s):
    h = s["hyper"]
    g, p = s["g"].double(), s["p"].double()
    if c["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m = (s["m"].double().view(-1, BLOCK) * s["m_scale"].double()[:, None]).flatten()
        v = (s["v"].double().view(-1, BLOCK) * s["v_scale"].double()[:, None]).flatten() ** 2
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    update = (m / (1 - h["beta1"] ** h["step"])) / ((v / (1 - h["beta2"] ** h["step"])).sqrt() + h["eps"])
    for (n, _), o, d in zip(s["sizes"], s["off"], s["decay"]):
        p[o:o + n] *= 1 - h["lr"] * d
    p = p - h["lr"] * update
    out = dict(p=p, m=m, v=v)
    if c["copy"]:
        out["copy"] = p
    if c["bits"] == 8:       # which neighbour a value goes to is the random bits' choice
        out["m"] = out["v"] = None
        out["m_scale"] = m.view(-1, BLOCK).abs().amax(1) / 448
        out["v_scale"] = v.sqrt().view(-1, BLOCK).amax(1) / 448
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("attn"):
        return _exact_attention(case, s)
    return _exact_loss(case, s) if case["kind"].startswith("loss") else _exact_adamw(case, s)
