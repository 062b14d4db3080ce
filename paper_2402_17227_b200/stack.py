"""Backward pass through a stack of linear layers with the chain entry point (vcas_linear_bwd_chain), from a loss over
tokens, through the attention between two of them, to the optimizer step.

Orchestration only: which layer hands what to the next one.  Going down the stack (the order of
backpropagation) every layer receives the list of data the layer above kept - all other data have an
all-zero gradient by then (Sec. 4: the activation gradient gets sparser from layer to layer) - and, when its
incoming gradient is the previous layer's dX, that gradient's row square-norms from the producer's epilogue.
Every step of the method itself runs inside the library's kernels.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as vb


@dataclass
class TokenLossInput:
    """The loss on top of a stack: what the forward pass left for its gradient, one of each per batch variant.

    logits: [R, vocab] (rows may be padded); tokens: [R], negative where there is none; g_logp, g_entropy: the loss's
    derivatives by logp and entropy ([R] float32; -1/R for a mean cross-entropy)."""
    op: vb.TokenLoss
    logits: list
    tokens: list
    lse: list
    g_logp: list
    entropy: list | None = None
    g_entropy: list | None = None


@dataclass
class AttentionInput:
    """An attention between two layers of a stack: q, k and v as the layer under it made them, side by side in [R, heads_q +
    2 heads_kv, head_dim], and what its forward pass left, one of each per batch variant.  starts: int32 [N + 1], the N data of T
    tokens each: 0, T, .., N T."""
    op: vb.Attention
    qkv: list
    o: list
    lse: list
    starts: torch.Tensor

    def split(self, x):
        """q, k and v (or their gradients) in a [R, heads_q + 2 heads_kv, head_dim] buffer."""
        hq, hk = self.op.heads_q, self.op.heads_kv
        return x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]


@dataclass
class StackLayer:
    """One linear layer of the stack, in backward order.

    dY: the incoming gradients that a layer is given, and on which it is probed.  One that gets its gradient from the layer above or
    from a loss needs none: it is then probed on the exact gradients of the batch variants.
    chained: this layer's dY is the dX of the layer before it in backward order.
    attention: this layer's dY is the gradient of an attention whose output is the input of the layer before it in backward
    order.
    loss: this layer's dY is the gradient of a loss over tokens (the first layer in backward order); d_out may exceed the
    vocabulary, the gradient is 0 there.
    H: pre-activation of a GELU feeding THIS layer's input; its dX is multiplied by GELU'(H) (App. E)."""
    name: str
    d_in: int
    d_out: int
    W: torch.Tensor
    X: list            # input activations, one tensor per batch variant [R, d_in]
    dY: list           # incoming gradients per batch variant [R, d_out]
    H: list | None = None      # pre-activation of the GELU feeding this layer's input, per variant [R, d_in]
    chained: bool = False
    attention: AttentionInput | None = None
    loss: TokenLossInput | None = None
    handle: vb.Layer | None = None
    kept: torch.Tensor | None = None
    kept_cnt: torch.Tensor | None = None
    a_out: torch.Tensor | None = None
    dX: torch.Tensor | None = None
    dW: torch.Tensor | None = None
    grad: torch.Tensor | None = None       # dY of a layer with attention or loss
    norms: torch.Tensor | None = None      # its rows' square-norms, from the loss


class LinearStack:
    """Owns the per-layer outputs and runs one backward pass per call of `backward`.

    Handles are shared between layers of the same shape (a handle's workspace serves one call at a time and
    the calls of a pass follow one another on one stream)."""

    def __init__(self, layers: list[StackLayer], N: int, T: int, dtype=torch.bfloat16, config=None,
                 gemm_path: int = vb.GEMM_AUTO, skip_dropped_rows: bool = False, overlap_layers: bool = False):
        """skip_dropped_rows: the rows of dX that belong to dropped data are not written (every consumer in the
        stack takes the kept-data list and never reads them); the dX buffers then hold stale rows there."""
        self.layers, self.N, self.T, self.dtype = layers, N, T, dtype
        self.skip_dropped_rows = skip_dropped_rows
        # overlap_layers: a layer's weight-gradient branch is left running while the next layers are scored and
        # their dX products run (vcas_chain_args::defer_join); all handles are joined at the end of the pass
        self.overlap_layers = overlap_layers
        self.R = N * T
        self.handles: dict = {}
        dev = layers[0].W.device
        for i, L in enumerate(layers):
            key = (L.d_in, L.d_out)
            if key not in self.handles:
                self.handles[key] = vb.Layer(N, T, L.d_in, L.d_out, dtype, gemm_path, config)
            L.handle = self.handles[key]
            L.kept = torch.zeros(N, dtype=torch.int32, device=dev)
            L.kept_cnt = torch.zeros(1, dtype=torch.int32, device=dev)
            L.dW = torch.empty(L.d_out, L.d_in, dtype=torch.float32, device=dev)
            assert (L.loss is None or i == 0) and (L.attention is None or i > 0) and \
                sum((L.chained, L.attention is not None, L.loss is not None)) <= 1, "one source of a layer's dY"
            if L.attention is not None:
                a = L.attention.op
                assert layers[i - 1].d_in == a.heads_q * a.head_dim and L.d_out == (a.heads_q + 2 * a.heads_kv) * a.head_dim
                if L.attention.starts.shape != (N + 1,) or L.attention.starts.tolist() != [n * T for n in range(N + 1)]:
                    raise ValueError(f"{L.name}: starts of an attention in a stack are those of the {N} data of {T} tokens")
                L.grad = torch.empty(self.R, L.d_out, dtype=dtype, device=dev)
            if L.loss is not None:
                assert L.loss.op.vocab <= L.d_out
                L.grad = torch.zeros(self.R, L.d_out, dtype=dtype, device=dev)
                L.norms = torch.empty(self.R, dtype=torch.float32, device=dev)
            nxt = layers[i + 1] if i + 1 < len(layers) else None
            if nxt is not None and nxt.chained:
                assert nxt.d_out == L.d_in, "a chained layer's dY is the previous layer's dX"
                L.dX = torch.empty(self.R, L.d_in, dtype=dtype, device=dev)          # kept: it is the next layer's dY
                L.a_out = torch.empty(self.R, L.handle.chain_parts(), dtype=torch.float32, device=dev)
        # layers whose dX nobody consumes write into one scratch buffer per width
        self._scratch = {}
        for L in layers:
            if L.dX is None:
                if L.d_in not in self._scratch:
                    self._scratch[L.d_in] = torch.empty(self.R, L.d_in, dtype=dtype, device=dev)
                L.dX = self._scratch[L.d_in]

    def backward(self, rho, nu, seed: int, variant: int = 0, hook=None) -> None:
        """One sampled backward pass, top layer first.  rho, nu: per-layer keep ratios in backward order.
        hook(i, layer, after): optional callback before (after=False) and after every layer's call."""
        prev = None
        for i, L in enumerate(self.layers):
            v = variant % len(L.X)
            kw = {}
            if prev is not None:
                kw.update(alive_in=prev.kept, alive_cnt_in=prev.kept_cnt)
            if hook is not None:
                hook(i, L, False)
            if L.chained:
                dY = prev.dX
                kw.update(a_in=prev.a_out, a_in_parts=prev.handle.chain_parts())
            elif L.attention is not None:
                dY = self._attention_grad(L, prev.dX, v, alive_in=prev.kept, alive_cnt_in=prev.kept_cnt,
                                          skip_dropped_rows=self.skip_dropped_rows)
            elif L.loss is not None:
                dY = self._loss_grad(L, v)
                kw.update(a_in=L.norms, a_in_parts=1)
            else:
                dY = L.dY[v]
            H = L.H[v % len(L.H)] if L.H is not None else None
            L.handle.linear_bwd_chain(L.X[v], dY, L.W, float(rho[i]), float(nu[i]), seed * len(self.layers) + i,
                                      L.dX, L.dW, H=H, a_out=L.a_out, kept_out=L.kept, kept_cnt_out=L.kept_cnt,
                                      skip_dropped_rows=self.skip_dropped_rows, defer_join=self.overlap_layers, **kw)
            if hook is not None:
                hook(i, L, True)
            prev = L
        if self.overlap_layers:
            for h in self.handles.values():
                h.join()

    def _attention_grad(self, L: StackLayer, dO: torch.Tensor, v: int, out=None, **kept):
        """dY of the layer under an attention from the dX of the layer above it; of the kept data only, where they are given."""
        a, out = L.attention, L.grad if out is None else out
        q, k, vv = a.split(a.qkv[v])
        dq, dk, dv = a.split(out.view(self.R, -1, a.op.head_dim))
        a.op.bwd(dO.view(a.o[v].shape), q, k, vv, a.o[v], a.lse[v], a.starts, dq=dq, dk=dk, dv=dv, **kept)
        return out

    def _loss_grad(self, L: StackLayer, v: int, out=None, norms=None):
        """dY of the top layer, and its rows' square-norms."""
        o, out = L.loss, L.grad if out is None else out
        o.op.bwd(o.logits[v], o.tokens[v], o.lse[v], o.g_logp[v], entropy=o.entropy[v] if o.entropy else None,
                 g_entropy=o.g_entropy[v] if o.g_entropy else None, dlogits=out[:, :o.op.vocab], a_out=L.norms if norms is None else norms)
        return out

    def make_optimizer(self, bits: int = 32, weight_decay: float = 0.0) -> vb.AdamW:
        """AdamW over the stack's weights from their dW, in one launch: fp32 weights in place; bf16 ones from fp32 masters that the
        optimizer holds (its `tensors[i].p`), the bf16 weights being the copy that each step writes.  bits: of the states."""
        entries = []
        for L in self.layers:
            low = L.W.dtype == torch.bfloat16
            entries.append(vb.AdamWTensor.make(L.W.float() if low else L.W, L.dW, bits, copy=L.W if low else None,
                                               weight_decay=weight_decay))
        return vb.AdamW(entries)

    def dense_backward(self, variant: int = 0, hook=None) -> None:
        """The exact backward of the same layers (no sampling; the GELU Jacobian where the sampled pass has it):
        the dense comparison."""
        prev = None
        for i, L in enumerate(self.layers):
            v = variant % len(L.X)
            if hook is not None:
                hook(i, L, False)
            if L.attention is not None:
                dY = self._attention_grad(L, prev.dX, v)
            elif L.loss is not None:
                dY = self._loss_grad(L, v)
            else:
                dY = prev.dX if L.chained else L.dY[v]
            H = L.H[v % len(L.H)] if L.H is not None else None
            L.handle.dense_bwd(L.X[v], dY, L.W, H=H, dX=L.dX, dW=L.dW)
            if hook is not None:
                hook(i, L, True)
            prev = L

    def _exact_grads(self) -> list:
        """Every layer's dY in every batch variant: the ones it was given, else those of an exact pass down the stack.  What
        `backward` left (dW, dX, grad) stays as it is."""
        M = len(self.layers[0].X)
        if any(len(L.X) != M for L in self.layers):
            raise ValueError("layers of one stack with different numbers of batch variants")
        new = lambda *shape, dt=self.dtype: torch.zeros(*shape, dtype=dt, device=self.layers[0].W.device)
        grads = [[] for _ in self.layers]
        for v in range(M):
            dX = None                    # of the layer above, where this one takes it
            for i, L in enumerate(self.layers):
                if L.dY:
                    dY = L.dY[v]
                elif L.chained:
                    dY = dX
                elif L.attention is not None:
                    dY = self._attention_grad(L, dX, v, new(self.R, L.d_out))
                elif L.loss is not None:
                    dY = self._loss_grad(L, v, new(self.R, L.d_out), new(self.R, dt=torch.float32))
                else:
                    raise ValueError(f"{L.name}: no gradient to probe it on")
                grads[i].append(dY)
                below = self.layers[i + 1] if i + 1 < len(self.layers) else None
                if below is not None and not below.dY and (below.chained or below.attention is not None):
                    dX, _ = L.handle.dense_bwd(L.X[v], dY, L.W, H=L.H[v % len(L.H)] if L.H is not None else None)
        return grads

    def probe(self, rho, nu, s: float, seed: int):
        """Alg. 1's probe for every layer (M = number of batch variants).  Returns a [L, 5] device tensor of
        (V_s, V_act, V_w, p_lo, p_hi).  A layer is probed on its own gradient variants `dY`; where it has none because its gradient comes
        from the layer above it or from a loss, on the exact gradients of the variants."""
        dev = self.layers[0].W.device
        out = torch.zeros(len(self.layers), 5, dtype=torch.float32, device=dev)
        grads = [L.dY for L in self.layers] if all(L.dY for L in self.layers) else self._exact_grads()
        for i, L in enumerate(self.layers):
            L.handle.variance_probe(L.X, grads[i], L.W, float(rho[i]), float(nu[i]), float(s), seed + i, out=out[i])
        return out

    def workspace_bytes(self) -> int:
        return sum(h.workspace_bytes() for h in self.handles.values())

    def device_status(self) -> int:
        """The first status that is not VCAS_OK of the stack's handles, its attentions' and its loss's among them; all are cleared."""
        ops = list(self.handles.values()) + [o.op for L in self.layers for o in (L.attention, L.loss) if o is not None]
        return next((st for st in [op.device_status() for op in ops] if st != 0), 0)

    def close(self) -> None:
        for h in self.handles.values():
            h.close()
        self.handles = {}
