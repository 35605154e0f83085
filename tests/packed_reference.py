"""Attention over packed sequences in 64 bits, with its gradients, and how far a right implementation may be off:
every rounding counted at half a step of its type, first order, on the sums of absolute values."""
from __future__ import annotations

import math

import numpy as np
import torch

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def offsets(lens):
    return [0] + [int(x) for x in np.cumsum(lens)]


def visible(nq, nk):
    return torch.ones(nq, nk, dtype=torch.bool).tril(nk - nq)


def sequence(q, k, v, g, scale, dtype):
    """One head of one sequence (64 bits, CPU): {name: (value, bound)}.  g: gradient of the output, or None."""
    nq, d = q.shape
    nk = k.shape[0]
    see, h = visible(nq, nk), HALF[dtype]
    s = torch.where(see, scale * (q @ k.T), -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.where(see, torch.exp(s - lse[:, None]), 0.0)
    out = p @ v
    # a score: d products and sums, the scale, the base-2 exponent's fused multiply and its result
    es = U * ((d + 4) * abs(scale) * (q.abs() @ k.abs().T) + 4 * torch.where(see, s.abs(), 0.0) + 8)
    worst = torch.where(see, es, 0.0).amax(1, keepdim=True) if nk else torch.zeros(nq, 1, dtype=torch.float64)
    ep = torch.where(see, es + worst + U * (nk + 8), 0.0)          # relative, of a weight in fp32
    a = p @ v.abs()
    # the numerator sees the rounded weight, the denominator the one in fp32; nk sums; the result's own rounding
    bo = (p * (h + 2 * ep + 2 * nk * U)) @ v.abs() + h * out.abs() + 2 * U * a
    got = {"out": (out, bo), "lse": (lse, torch.where(torch.isinf(lse), 0.0, worst[:, 0] + (nk + 16) * U + 4 * U * lse.abs()))}
    if g is not None:
        dp = g @ v.T
        delta = (g * out).sum(1, keepdim=True)
        edp = U * (d + 2) * (g.abs() @ v.abs().T)
        edelta = (g.abs() * (bo + h * out.abs())).sum(1, keepdim=True) + U * (d + 2) * (g.abs() * out.abs()).sum(1, keepdim=True)
        t = p * (dp - delta)
        elp = ep + got["lse"][1][:, None]                           # the weight, taken again from the stored lse
        et = p * (edp + edelta + elp * (dp - delta).abs()) + (h + 3 * U) * t.abs()
        n = nk + nq
        dq, dk, dv = scale * t @ k, scale * t.T @ q, p.T @ g
        got["dq"] = (dq, abs(scale) * (et + n * U * t.abs()) @ k.abs() + (h + U) * dq.abs())
        got["dk"] = (dk, abs(scale) * (et + n * U * t.abs()).T @ q.abs() + (h + U) * dk.abs())
        got["dv"] = (dv, (p * (h + elp + n * U)).T @ g.abs() + (h + U) * dv.abs())
    return got


def packed(q, k, v, g, lens_q, lens_k, scale, dtype):
    """The same for [rows, heads, d]; rows behind the last sequence are zero."""
    q, k, v = (x.detach().double().cpu() for x in (q, k, v))
    g = None if g is None else g.detach().double().cpu()
    H, G = q.shape[1], q.shape[1] // k.shape[1]
    zero = lambda x: [torch.zeros_like(x), torch.zeros_like(x)]
    full = {"out": zero(q), "lse": zero(q[:, :, 0].T.contiguous()), "dq": zero(q), "dk": zero(k), "dv": zero(k)}
    cq, ck = offsets(lens_q), offsets(lens_k)
    for s in range(len(lens_q)):
        a, c = slice(cq[s], cq[s + 1]), slice(ck[s], ck[s + 1])
        for h in range(H):
            got = sequence(q[a, h], k[c, h // G], v[c, h // G], None if g is None else g[a, h], scale, dtype)
            for name, pair in got.items():
                for to, x in zip(full[name], pair):
                    if name == "lse":
                        to[h, a] = x
                    elif name in ("dk", "dv"):
                        to[c, h // G] += x
                    else:
                        to[a, h] = x
    return full


def check(got, want, bound, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, what
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, 0.0, (got - want).abs())
    bad = ~(off <= bound + 1e-30)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} values are off, first at {bad.nonzero()[0].tolist()}: "
                           f"{got[bad][0].item()} for {want[bad][0].item()}, allowed {bound[bad][0].item():.3g}")
    return float((off / bound.clamp(min=1e-30)).max()) if off.numel() else 0.0
