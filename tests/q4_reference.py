"""Rows of 4 bits a value, and attention over them, in 64 bits (numpy and torch on the CPU), with how far a right implementation may
be off: every rounding counted at half a step of its type, first order, on the sums of absolute values."""
from __future__ import annotations

import math

import numpy as np
import torch

from tests.packed_reference import HALF, TYPES, U  # noqa: F401


def _bits(x):
    """bf16 patterns of finite values that are bf16 values already."""
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def _grid(x, to):
    """x moved by `to` onto bf16's values: 8 significant bits, the smallest step 2^-133."""
    _, e = np.frexp(x)
    unit = np.exp2(np.maximum(e - 8.0, -133.0))
    return to(x / unit) * unit


def quantise(x):
    """[..., d] values (torch) -> (codes [..., d], scale [..., d / 32], low [..., d / 32]), 64 bits."""
    x = x.detach().double().cpu().numpy()
    g = x.reshape(*x.shape[:-1], -1, 32)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        sound = (np.abs(g) < 2.0 ** 127).all(-1)
        g = np.where(sound[..., None], g, 0.0)
        low = _grid(g.min(-1), np.floor) + 0.0             # zero without its sign
        scale = _grid((g.max(-1) - low) / 15.0, np.ceil)
        at = np.where(scale[..., None] > 0, (g - low[..., None]) / scale[..., None], 0.0)
    codes = np.rint(at)                                     # half to even
    assert codes.min(initial=0) >= 0 and codes.max(initial=0) <= 15
    nan = np.where(sound, 0.0, np.nan)
    return codes.reshape(x.shape), scale + nan, low + nan


def rows(x):
    """[..., d] values -> the bytes that hold them [..., d / 2 + d / 8]."""
    codes, scale, low = quantise(x)
    d = codes.shape[-1]
    n = codes.astype(np.uint8)
    out = np.zeros((*codes.shape[:-1], d // 2 + d // 8), np.uint8)
    out[..., :d // 2] = n[..., 0::2] | n[..., 1::2] << 4
    pair = np.stack([scale, low], -1)
    bits = np.where(np.isnan(pair), np.uint16(0x7fc0), _bits(np.where(np.isnan(pair), 0.0, pair)))
    out[..., d // 2:] = bits.reshape(*codes.shape[:-1], -1).view(np.uint8)
    return torch.from_numpy(out)


def parts(rows_):
    """Bytes -> (codes [..., d], scale, low [..., d]: each channel's), 64 bits (torch)."""
    r = rows_.cpu().numpy()
    d = r.shape[-1] * 8 // 5
    codes = np.zeros((*r.shape[:-1], d))
    codes[..., 0::2], codes[..., 1::2] = r[..., :d // 2] & 15, r[..., :d // 2] >> 4
    pair = np.ascontiguousarray(r[..., d // 2:]).view(np.uint16).astype(np.uint32) << 16
    with np.errstate(invalid="ignore"):
        pair = pair.view(np.float32).astype(np.float64).reshape(*r.shape[:-1], d // 32, 2)
    return tuple(torch.from_numpy(x) for x in (codes, np.repeat(pair[..., 0], 32, -1), np.repeat(pair[..., 1], 32, -1)))


def values(rows_):
    codes, scale, low = parts(rows_)
    return low + scale * codes


def one_head(q, krows, vrows, scale, dtype):
    """One query [d] over rows of bytes: (output, bound), 64 bits."""
    h, d, n = HALF[dtype], q.numel(), krows.shape[0]
    if n == 0:
        return torch.zeros(d, dtype=torch.float64), torch.zeros(d, dtype=torch.float64)
    kc, ks, kl = parts(krows)
    vc, vs, vl = parts(vrows)
    x = scale * ((kl + ks * kc) @ q)
    p = torch.softmax(x, 0)
    out = p @ (vl + vs * vc)
    # a score: products of codes and queries are exact; a group's 32, in up to three parts, are summed in a matrix product whose
    # additions may cut (two half steps), the query's own sum of 32 likewise; then the pair's fused product, up to four groups, the
    # scale and the base-2 exponent
    size = abs(scale) * ((ks * kc + kl.abs()) @ q.abs())
    es = 2 * U * (3 * 32 + 16) * size + U * (4 * x.abs() + 8)
    ep = es + es.max() + U * (n + 8)                          # relative, of a weight in fp32
    held = vl.abs() + vs * vc
    # the weight times its scale is rounded (bf16) or taken in parts to 24 bits; n sums whose additions may cut; the result's rounding
    bound = (p * h) @ (vs * vc) + (p * (2 * ep + 4 * (n + 8) * U)) @ held + h * out.abs() + 4 * U * (p @ held)
    return out, bound


def decode(q, kpages, vpages, table, lens, page, scale, dtype, room, lone=None):
    """q [B, H, d]; pages of bytes as they are after the step; lens: tokens each row sees (None in its place: idle); lone: {row: bytes
    of its key and value} of new tokens that no page holds.  (output, bound) [B, H, d]."""
    B, H, d = q.shape
    Hkv = kpages.shape[1]
    q = q.detach().double().cpu()
    out, bound = torch.zeros(B, H, d, dtype=torch.float64), torch.zeros(B, H, d, dtype=torch.float64)
    kp, vp = kpages.cpu(), vpages.cpu()
    for b in range(B):
        if lens[b] is None or lens[b] > room:
            continue
        at = [(int(table[b, t // page]), t % page) for t in range(lens[b]) if 0 <= int(table[b, t // page]) < kp.shape[0]]
        ids, slots = torch.tensor([x[0] for x in at], dtype=torch.long), torch.tensor([x[1] for x in at], dtype=torch.long)
        for g in range(Hkv):
            kr, vr = kp[ids, g, slots], vp[ids, g, slots]
            if lone and b in lone:
                kr, vr = (torch.cat([x, y[g:g + 1]]) for x, y in zip((kr, vr), lone[b]))
            for h in range(g * H // Hkv, (g + 1) * H // Hkv):
                out[b, h], bound[b, h] = one_head(q[b, h], kr, vr, scale, dtype)
    return out, bound
