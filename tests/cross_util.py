"""Attention over keys of another length and over shared keys, in 64 bits from the
definition, with bounds on what the kernels may be off (CPU or GPU tensors).

Bounds.  A rounding to bf16 is off by at most u = 2^-8 of the value.  The kernels
round P (before P V and P^T dO), dS (before dS K and dS^T Q) and their outputs, and
take D = <dO, O> from the rounded O; everything else is 32 bits, whose errors (a
logit is off by at most about d 2^-24 sum |q k|) the factor SLACK covers for the
logits of these tests.  So, element by element:
  |dO_i| <= u (|O_i| + sum_j P_ij |v_j|)
  |d dV| <= u (sum P |dO| + |dV|),  |d D_i| <= sum |dO_i| (bound of O_i)
  |d dK| <= scale (u |dS| + P |d D|)^T |Q| + u |dK|,  dQ the same way
(the last term only where the gradient is written in bf16)."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -8
SLACK = 1.05
TINY = 1e-6


def offsets(lengths, device="cpu"):
    c = [0]
    for x in lengths:
        c.append(c[-1] + x)
    return torch.tensor(c, dtype=torch.int32, device=device)


def visible(nq, nk, causal, device):
    """[nq, nk] whether query i sees key j; causal: the last query sees every key."""
    i, j = torch.arange(nq, device=device), torch.arange(nk, device=device)
    see = torch.ones((nq, nk), dtype=torch.bool, device=device)
    return see & (j[None] <= i[:, None] + nk - nq) if causal else see


def reference(q, k, v, cu_q, cu_k, causal, scale, used=None, kp=None, vp=None, do=None):
    """{name: (value, bound)} of o, lse and, with do, dq, dk, dv (dkp, dvp) in 64 bits;
    bounds without an output's own rounding, but for o."""
    dev = q.device
    cu_q, cu_k = cu_q.tolist(), cu_k.tolist()
    hq, hkv = q.shape[1], k.shape[1] if k.shape[0] or kp is None else kp.shape[1]
    g, p = hq // hkv, 0 if kp is None else kp.shape[0]
    f = {n: t.double() for n, t in dict(q=q, k=k, v=v, kp=kp, vp=vp, do=do).items()
         if t is not None}

    def zeros(t):
        return torch.zeros(t.shape, dtype=torch.float64, device=dev)

    out = {"o": (zeros(q), zeros(q))}
    lse = torch.full((hq, q.shape[0]), -math.inf, dtype=torch.float64, device=dev)
    out["lse"] = (lse, torch.zeros_like(lse))
    if do is not None:
        for n in ("q", "k", "v") + (("kp", "vp") if p else ()):
            out["d" + n] = (zeros(f[n]), zeros(f[n]))
    for s in range(len(cu_q) - 1):
        a, b, c = cu_q[s], cu_q[s + 1], cu_k[s]
        nk = cu_k[s + 1] - c if used is None else int(used[s])
        nq = b - a
        see = torch.cat([torch.ones((nq, p), dtype=torch.bool, device=dev),
                         visible(nq, nk, causal, dev)], 1)
        for h in range(hq):
            e = h // g
            Q = f["q"][a:b, h]
            K, V = f["k"][c:c + nk, e], f["v"][c:c + nk, e]
            if p:
                K, V = torch.cat([f["kp"][:, e], K]), torch.cat([f["vp"][:, e], V])
            S = (Q @ K.T * scale).masked_fill(~see, -math.inf)
            L = torch.logsumexp(S, 1) if S.shape[1] else torch.full((nq,), -math.inf, device=dev,
                                                                    dtype=torch.float64)
            P = torch.exp(S - torch.where(L == -math.inf, 0.0, L)[:, None])
            O = P @ V
            dO = SLACK * U * (O.abs() + P @ V.abs()) + TINY
            out["o"][0][a:b, h], out["o"][1][a:b, h] = O, dO
            lse[h, a:b] = L
            logit = scale * q.shape[2] * 2.0 ** -24 * (Q.abs() @ K.abs().T).amax(1) \
                if S.shape[1] else torch.zeros_like(L)
            out["lse"][1][h, a:b] = logit + 2.0 ** -21 * (1 + L.abs())
            if do is None:
                continue
            G = f["do"][a:b, h]
            D = (G * O).sum(1, keepdim=True)
            dS = P * (G @ V.T - D)
            edS = U * dS.abs() + P * (G.abs() * dO).sum(1, keepdim=True)
            out["dq"][0][a:b, h] = scale * (dS @ K)
            out["dq"][1][a:b, h] = SLACK * scale * (edS @ K.abs()) + TINY
            for name, val, err in (("k", scale * (dS.T @ Q), scale * (edS.T @ Q.abs())),
                                   ("v", P.T @ G, U * (P.T @ G.abs()))):
                err = SLACK * err + TINY
                out["d" + name][0][c:c + nk, e] += val[p:]
                out["d" + name][1][c:c + nk, e] += err[p:]
                if p:
                    out["d" + name + "p"][0][:, e] += val[:p]
                    out["d" + name + "p"][1][:, e] += err[:p]
    return out


def check(name, got, want, rows=None):
    """Every element within its bound (rows: only those of the first dimension)."""
    val, bound = want
    if rows is not None:
        got, val, bound = got[rows], val[rows], bound[rows]
    if name != "o" and got.dtype == torch.bfloat16:
        bound = bound + U * val.abs()
    x = got.double()
    same = (x == val) | (torch.isnan(x) & torch.isnan(val))
    off = torch.where(same, 0.0, (x - val).abs() / bound.clamp_min(1e-30))
    off = torch.where(torch.isnan(off), math.inf, off)
    worst = float(off.max()) if off.numel() else 0.0
    print(f"    {name:4s} worst {worst:.3f} of its bound (n={off.numel()})", flush=True)
    assert worst <= 1.0, f"{name}: {worst:.3g} times its bound at {int(off.argmax())}"
