"""Attention and its gradients in 64 bits on the host, written from the
definition, with bounds of what a correct kernel may differ by."""
from __future__ import annotations

import math

import torch

# Unit roundoff of a type: half the distance of 1 to the next number.
UNIT = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
# Largest absolute rounding error below the type's normal range.
TINY = {torch.float32: 0.0, torch.float16: 2.0**-25, torch.bfloat16: 0.0}


def visible(Tq, Tk, tq, tk, causal=False, doc_start=None, prefix=None):
    """[Tq, Tk] of one item: which key each query sees, and their distance."""
    i, j = torch.arange(Tq)[:, None], torch.arange(Tk)[None]
    place = i + (tk - tq)
    see = (i < tq) & (j < tk)
    free = torch.zeros((1, Tk), dtype=torch.bool)
    if doc_start is None:
        if prefix is not None:
            free = j < max(prefix[0], 0)
    else:
        same = torch.zeros((Tq, Tk), dtype=torch.bool)
        for n in range(len(doc_start) - 1):
            lo, hi = doc_start[n], doc_start[n + 1]
            same |= ((place >= lo) & (place < hi)) & ((j >= lo) & (j < hi))
            if prefix is not None:
                free = free | ((j >= lo) & (j < min(lo + max(prefix[n], 0), hi)))
        see &= same
    if causal:
        see &= (j <= place) | free
    return see, (place - j).abs().double()


def reference(q, k, v, dout=None, t_q=None, t_k=None, causal=False, scale=None, cap=0.0, slope=None, doc_start=None,
              prefix=None):
    """{name: (value, bound)} of out, lse and, with dout, dq, dk, dv.

    The bounds follow the operations: 16-bit p and ds are rounded once each
    (UNIT), results once; scores are fp32 dot products of D terms and a few more
    operations, and an absolute error e of a score is a relative error e of p;
    sums of n terms in fp32 err by n units at most; delta is formed from the
    rounded output.
    """
    dtype = q.dtype
    u, tiny, f32 = UNIT[dtype], TINY[dtype], UNIT[torch.float32]
    half = 0.0 if dtype == torch.float32 else u
    q, k, v = (x.cpu() for x in (q, k, v))
    B, Tq, Hq, D = q.shape
    Tk, Hk = k.shape[1], k.shape[2]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    host = lambda x: None if x is None else x.cpu().tolist()
    t_q, t_k, doc_start, prefix, slope = (host(x) for x in (t_q, t_k, doc_start, prefix, slope))
    new = lambda *s: torch.zeros(s, dtype=torch.float64)
    names = ["out"] + (["dq", "dk", "dv"] if dout is not None else [])
    shapes = {"out": q.shape, "dq": q.shape, "dk": k.shape, "dv": v.shape}
    res = {n: (new(*shapes[n]), new(*shapes[n])) for n in names}
    lse, lse_tol = torch.full((B, Hq, Tq), -math.inf, dtype=torch.float64), new(B, Hq, Tq)
    for b in range(B):
        tq = Tq if t_q is None else min(max(t_q[b], 0), Tq)
        tk = Tk if t_k is None else min(max(t_k[b], 0), Tk)
        see, distance = visible(Tq, Tk, tq, tk, causal, None if doc_start is None else doc_start[b],
                                None if prefix is None else prefix[b])
        for h in range(Hq):
            hk = h // (Hq // Hk)
            # Padding may hold anything: it is not part of the problem.
            Q, K, V = (torch.where((torch.arange(x.shape[1]) < n)[:, None], x[b, :, i].double(), 0.0)
                       for x, n, i in ((q, tq, h), (k, tk, hk), (v, tk, hk)))
            raw = Q @ K.T * scale
            s, bend = raw, torch.ones_like(raw)
            size = (Q.abs() @ K.abs().T) * abs(scale)
            if cap:
                t = torch.tanh(raw / cap)
                s, bend = cap * t, 1 - t * t
            if slope is not None:
                s = s - slope[h] * distance
            s = s.masked_fill(~see, -math.inf)
            any_seen = see.any(1)
            m = torch.where(any_seen, s.amax(1), 0.0)
            e = torch.exp(s - m[:, None])
            total = e.sum(1)
            p = e / total.clamp(min=1e-300)[:, None]
            # Error of a score, and so relative error of p (numerator and total).
            es = (D + 8) * f32 * size + 16 * f32 * (s.masked_fill(~see, 0.0).abs() + (cap or 0.0)
                                                    + (0.0 if slope is None else slope[h] * distance))
            ep = 2 * es.masked_fill(~see, 0.0).amax(1, keepdim=True) + (16 + Tk) * f32
            o = p @ V
            res["out"][0][b, :, h] = o
            res["out"][1][b, :, h] = u * o.abs() + ((half + ep) * p + tiny * see) @ V.abs()
            lse[b, h] = torch.where(any_seen, m + torch.log(total.clamp(min=1e-300)), -math.inf)
            lse_tol[b, h] = torch.where(any_seen, ep[:, 0] + 8 * f32 * lse[b, h].abs().clamp(max=1e6) + 8 * f32, 0.0)
            if dout is None:
                continue
            G = torch.where((torch.arange(Tq) < tq)[:, None], dout[b, :, h].cpu().double(), 0.0)
            dp = G @ V.T
            delta = (G * o).sum(1, keepdim=True)
            ds = p * (dp - delta) * bend
            # dp and delta are sums of D products; delta takes the rounded output.
            span = G.abs() @ V.abs().T + (G.abs() * o.abs()).sum(1, keepdim=True)
            off = u * (G.abs() * o.abs()).sum(1, keepdim=True) + (G.abs() * res["out"][1][b, :, h]).sum(1, keepdim=True)
            ds_err = half * ds.abs() + tiny * see + p * (off + (ep + (2 * D + 32) * f32) * span)
            p_err = (half + ep) * p + tiny * see
            n = (16 + max(Tk, Tq * (Hq // Hk))) * f32
            for name, at, value, err in (
                ("dq", (b, slice(None), h), scale * ds @ K, abs(scale) * (ds_err + n * ds.abs()) @ K.abs()),
                ("dk", (b, slice(None), hk), scale * ds.T @ Q, abs(scale) * (ds_err + n * ds.abs()).T @ Q.abs()),
                ("dv", (b, slice(None), hk), p.T @ G, (p_err + n * p).T @ G.abs())):
                res[name][0][at] += value
                res[name][1][at] += err
    for name in names[1:]:
        res[name][1].add_(u * res[name][0].abs())
    # Results below the normal range round to their type's absolute unit too.
    for name in names:
        res[name][1].add_(tiny + 1e-30)
    res["lse"] = (lse, lse_tol)
    return res


def check(got, want, what):
    value, bound = want
    got = got.detach().cpu().double()
    assert got.shape == value.shape, what
    same = (got == value) | ((got - value).abs() <= bound)
    assert bool(same.all()), (f"{what}: {int((~same).sum())} of {same.numel()} off, first at "
                              f"{torch.nonzero(~same)[0].tolist()}, worst {((got - value).abs() / bound).nan_to_num(9e9)[~same].max():.3g} bounds")
