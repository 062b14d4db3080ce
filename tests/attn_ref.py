"""Attention over packed sequences in 64 bits from its formulas, with a bound on how far a correct kernel may be off.

Half a rounding step relative to the value is u = finfo(dtype).eps / 2.  A kernel may round P (and dS) to the layer's type where
they enter a product, and the result once; sums, scores and exponentials are fp32:
  - a score's exponent is off by |S| fp32 roundings of its D + 8 operations, so P is off by at most the factor
    `g` = 2^-24 (D + 8) max(s sum |q||k|) + 2^-21 (the latter for the exponential itself), the normalised one by 2 g;
  - a sum of n terms adds n 2^-24 of the sum of absolute terms;
  - delta = rowsum(dO O) inherits the rounding of the stored O: u sum |dO||O|, and its own sum's D 2^-24.
With `parts` = 2 the bounds are those of P and dS as sums of two numbers of the layer's type, the second the first's rounding error
(u of it) rounded in its turn, so that u^2 is left, and of delta = rowsum(P dP), which has P's factor and the errors of the two sums.
"""
import torch

F = 2.0 ** -24


def _one(q, k, v, causal, scale):
    S = (q @ k.T) * scale
    if causal:
        n = S.shape[0]
        S = S.masked_fill(torch.ones(n, n, dtype=torch.bool, device=S.device).triu(1), float("-inf"))
    lse = torch.logsumexp(S, 1)
    return torch.exp(S - lse[:, None]), lse


def reference(q, k, v, starts, causal, scale, do=None, alive=None, parts=1):
    """Returns {name: (value, bound)} of o and lse, and with do of dq, dk, dv (those of `alive` sequences only; the others 0)."""
    dt = q.dtype
    u = torch.finfo(dt).eps / 2
    uP = u ** parts if dt != torch.float32 else 0.0          # P and dS stay in fp32 there
    q, k, v = q.double(), k.double(), v.double()
    Hq, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    zeros = lambda x: (torch.zeros_like(x), torch.zeros_like(x))
    out = dict(o=zeros(q), dq=zeros(q), dk=zeros(k), dv=zeros(v))
    lse = torch.zeros(Hq, q.shape[0], dtype=torch.float64, device=q.device)
    out["lse"] = (lse, torch.zeros_like(lse))
    st = starts.tolist()
    for n in range(len(st) - 1):
        t, L = slice(st[n], st[n + 1]), st[n + 1] - st[n]
        if L == 0:
            continue
        for h in range(Hq):
            hk = h // (Hq // Hk)
            Q, K, V = q[t, h], k[t, hk], v[t, hk]
            P, l = _one(Q, K, V, causal, scale)
            A = float((Q.abs() @ K.abs().T).max()) * scale
            g = F * (D + 8) * A + 2.0 ** -21
            O = P @ V
            PV = P @ V.abs()
            out["o"][0][t, h] = O
            out["o"][1][t, h] = u * O.abs() * 1.01 + (uP * 1.01 + 3 * g + L * F) * PV
            out["lse"][0][h, t] = l
            out["lse"][1][h, t] = 2 * g + L * F + 2 * F * l.abs()
            if do is None or (alive is not None and n not in alive):
                continue
            dO = do[t, h].double()
            dP = dO @ V.T
            Or = O.to(dt).double()
            delta = (dO * Or).sum(1)
            dS = P * (dP - (dO * O).sum(1)[:, None])
            # off by: P's factor, delta (O's own rounding and its sum), dP's sum
            e_delta = (u * 1.01 + D * F) * (dO.abs() * O.abs()).sum(1)
            if parts == 2:
                e_delta = (3 * g + (L + D + 4) * F) * (P * (dO.abs() @ V.abs().T)).sum(1)
                delta = (dO * O).sum(1)
            e_dS = P * ((3 * g) * (dP - delta[:, None]).abs() + e_delta[:, None] + (D + 2) * F * (dO.abs() @ V.abs().T)) + 1.01 * uP * dS.abs()
            add = lambda name, at, value, bound: (out[name][0][at].add_(value), out[name][1][at].add_(bound))
            add("dv", (t, hk), P.T @ dO, (uP * 1.01 + 3 * g + L * F) * (P.T @ dO.abs()))
            add("dq", (t, h), scale * (dS @ K), scale * (e_dS @ K.abs() + (L + 2) * F * (dS.abs() @ K.abs())))
            add("dk", (t, hk), scale * (dS.T @ Q), scale * (e_dS.T @ Q.abs() + (L + 2) * F * (dS.abs().T @ Q.abs())))
    for name in ("dq", "dk", "dv"):                  # the result's own rounding; sums over a group of heads
        val, bound = out[name]
        bound.add_(u * 1.01 * val.abs() + (Hq // Hk) * F * val.abs())
    return out


def check(got, ref, rows=None, what=""):
    val, bound = ref
    got = got.double()
    if rows is not None:
        got, val, bound = got[rows], val[rows], bound[rows]
    assert torch.isfinite(got).all(), what
    over = ((got - val).abs() - bound * 1.001 - 1e-30)
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 0, (what, worst, float(((got - val).abs() / (bound + 1e-30)).max()))
