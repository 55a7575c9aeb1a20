"""A paged key/value cache in 64 bits from the definitions, with bounds on what the
kernels may be off (CPU or GPU tensors).

Bounds.  P is rounded to bf16 before the product with v, and o at the end, each off by at
most u = 2^-8 of the value: |dO_i| <= u (|O_i| + sum_j P_ij |v_j|).  Keys and values of an
e4m3 cache are exact in bf16, and their scales are applied in 32 bits.  A logit is a 32-bit
sum of d exact products, off by at most about d 2^-24 sum |q k|, and lse with it; a key's
weight is a sum of exp(S - lse), each off by the errors of S and lse and of an exponential
with an argument of their size, and is added to what was there in 32 bits."""
from __future__ import annotations

import math
import random

import torch

from tests.cross_util import SLACK, TINY, U, offsets, visible

E4M3 = torch.float8_e4m3fn


class Cache:
    """A pool in which the sequences' pages are anywhere; everything else in it, and in the
    table, is what no kernel may use: NaN, and pages that do not exist."""

    def __init__(self, lens, hkv, d, page, e4m3=False, device="cpu", seed=0, spare=3, extra=0,
                 values=None):
        g = torch.Generator().manual_seed(seed)
        rnd = random.Random(seed)
        used = [-(-n // page) for n in lens]
        self.page, self.hkv, self.d, self.e4m3, self.lens = page, hkv, d, e4m3, list(lens)
        pool = sum(used) + spare + extra * len(lens)
        order = list(range(pool))
        rnd.shuffle(order)
        width = max(used) + 2
        wild = [-1, pool, 1 << 30, -(1 << 31)]
        table = [[rnd.choice(wild) for _ in range(width)] for _ in lens]
        self.rows = []  # of a sequence: (page, place) of its keys
        at = 0
        for i, n in enumerate(used):
            table[i][:n] = order[at:at + n]
            at += n
            self.rows.append([(table[i][j // page], j % page) for j in range(lens[i])])
        self.new_table = torch.tensor([order[at + i * extra:at + (i + 1) * extra]
                                       for i in range(len(lens))], dtype=torch.int32,
                                      device=device).view(len(lens), extra)
        self.table = torch.tensor(table, dtype=torch.int32, device=device)
        self.len = torch.tensor(lens, dtype=torch.int32, device=device)
        shape = (pool, hkv, page, d)
        dtype = E4M3 if e4m3 else torch.bfloat16
        live = torch.zeros(pool, page, dtype=torch.bool)
        for r in self.rows:
            for p, s in r:
                live[p, s] = True
        self.live = live
        out = []
        for _ in range(2):
            x = torch.randn(shape, generator=g)
            if values is not None:
                x = values(x)
            x = (x / 0.02).clamp(-448, 448).to(E4M3) if e4m3 else x.to(dtype)
            bits = x.view(torch.uint8) if e4m3 else x.view(torch.int16)
            bits.masked_fill_(~live[:, None, :, None], 0x7f if e4m3 else 0x7fc0)
            out.append(x.to(device))
        self.k, self.v = out
        self.ks = self.vs = None
        if e4m3:
            self.ks = (torch.rand(hkv, generator=g) * 0.02 + 0.01).to(device)
            self.vs = (torch.rand(hkv, generator=g) * 0.02 + 0.01).to(device)
        # (any order of magnitude, equal ones, none)
        w = torch.exp(3 * torch.randn(shape[:3], generator=g))
        w = torch.where(torch.rand(shape[:3], generator=g) < 0.2, 0.25, w)
        w.masked_fill_(~live[:, None], math.nan)
        self.scores = w.to(device)

    def scales(self):
        return dict(k_scale=self.ks, v_scale=self.vs)

    def keys(self, i, h):
        """Keys and values of a sequence's head in 64 bits."""
        p = torch.tensor([x for x, _ in self.rows[i]], dtype=torch.long, device=self.k.device)
        s = torch.tensor([x for _, x in self.rows[i]], dtype=torch.long, device=self.k.device)
        out = []
        for x, scale in ((self.k, self.ks), (self.v, self.vs)):
            y = (x.view(torch.uint8)[p, h, s].view(E4M3) if self.e4m3 else x[p, h, s]).double()
            out.append(y if scale is None else y * scale[h].double())
        return out[0], out[1], p, s


def attention(c: Cache, q, lq, causal, scale):
    """{name: (value, bound)} of o, lse and the keys' weights (as scores, where in use)."""
    hq, g = q.shape[1], q.shape[1] // c.hkv
    dev, f64 = q.device, torch.float64
    o, eo = torch.zeros(q.shape, dtype=f64, device=dev), torch.zeros(q.shape, dtype=f64, device=dev)
    lse = torch.full((hq, q.shape[0]), -math.inf, dtype=f64, device=dev)
    el = torch.zeros_like(lse)
    w = torch.zeros(c.scores.shape, dtype=f64, device=dev)
    ew = torch.zeros_like(w)
    a = 0
    for i, nq in enumerate(lq):
        nk = c.lens[i]
        see = visible(nq, nk, causal, dev)
        for e in range(c.hkv):
            K, V, p, s = c.keys(i, e)
            for h in range(e * g, e * g + g):
                Q = q[a:a + nq, h].double()
                S = (Q @ K.T * scale).masked_fill(~see, -math.inf)
                L = torch.logsumexp(S, 1) if nk else torch.full((nq,), -math.inf, device=dev,
                                                                dtype=f64)
                P = torch.exp(S - torch.where(L == -math.inf, 0.0, L)[:, None])
                O = P @ V
                o[a:a + nq, h], eo[a:a + nq, h] = O, SLACK * U * (O.abs() + P @ V.abs()) + TINY
                lse[h, a:a + nq] = L
                if not nk or not nq:
                    continue
                logit = scale * c.d * 2.0 ** -24 * (Q.abs() @ K.abs().T).amax(1)
                size = torch.where(L == -math.inf, 0.0, L.abs())
                el[h, a:a + nq] = logit + 2.0 ** -21 * (1 + size)
                w[p, e, s] += P.sum(0)
                far = torch.where(see, S.abs(), 0.0)
                ew[p, e, s] += (P * (2 * logit[:, None] + 2.0 ** -20 * (1 + size[:, None] + far))).sum(0)
        a += nq
    return {"o": (o, eo), "lse": (lse, el),
            "scores": (w, ew + 2.0 ** -23 * (w + torch.nan_to_num(c.scores.double())) + 1e-12)}


def write(c: Cache, k, v, lq):
    """The pool after a write of packed k, v: (k, v, scores), bytes and all."""
    out = [c.k.clone(), c.v.clone(), c.scores.clone()]
    a = 0
    for i, nq in enumerate(lq):
        for t in range(nq):
            j = c.lens[i] - nq + t
            if j < 0:
                continue
            p, s = c.rows[i][j]
            for x, y, scale in ((out[0], k, c.ks), (out[1], v, c.vs)):
                row = y[a + t]
                if c.e4m3:
                    row = (row.float() / scale[:, None]).clamp(-448, 448).to(E4M3)
                    x.view(torch.uint8)[p, :, s] = row.view(torch.uint8)
                else:
                    x[p, :, s] = row
            out[2][p, :, s] = 0.0
        a += nq
    return out


def evict(c: Cache, budget, recent, first):
    """(kept, new lengths) of an eviction: key by key, the least goes, of equal ones the
    latest."""
    n = len(c.lens)
    kept = torch.full((n, c.hkv, budget), -1, dtype=torch.int32)
    for i, nk in enumerate(c.lens):
        for h in range(c.hkv):
            w = [float(c.scores[p, h, s]) for p, s in c.rows[i]]
            w = [-math.inf if math.isnan(x) else x for x in w]
            # (a NaN is below -inf)
            nan = [math.isnan(float(c.scores[p, h, s])) for p, s in c.rows[i]]
            stay = list(range(nk))
            if nk > budget:
                mid = sorted(range(first, nk - recent), key=lambda j: (nan[j], -w[j], j))
                mid = mid[:budget - first - recent]
                stay = sorted(list(range(first)) + mid + list(range(nk - recent, nk)))
            kept[i, h, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
    return kept, torch.tensor([min(x, budget) for x in c.lens], dtype=torch.int32)


def same_bits(x, y):
    if x.dtype == E4M3:
        return torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    kind = {2: torch.int16, 4: torch.int32}[x.element_size()]
    return torch.equal(x.view(kind), y.view(kind))


def queries(lq, hq, d, device="cpu", seed=0, spare=0):
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((sum(lq) + spare, hq, d), generator=g).to(torch.bfloat16)
    return q.to(device), offsets(lq, device)
