"""The precision that the 4-bit decode step states: weights times the values' scales to 16 bits in bf16 calls, to 24 in fp32 ones.  The bound
counts that, and no rounding of a weight to fewer bits, so that a step which kept fewer would not stay within it."""
from __future__ import annotations

import pytest
import torch

from paper_2412_19829_amd import binding as gb
from tests import packed_reference as pref
from tests import q4_reference as ref

gpu = pytest.mark.gpu
U = pref.U
KEPT = {"bf16": 16, "f32": 24}


def cut(x, bits):
    """To so many significant bits, half to even."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2.0 ** bits) / 2.0 ** bits, e)


def one_head(q, krows, vrows, scale, dtype, kept=None):
    """One query [d] over rows of bytes, in 64 bits: (output, bound), or with `kept` the output of a step that holds weights times scales in
    so many bits and is exact otherwise."""
    n, d = krows.shape[0], q.numel()
    kc, ks, kl = ref.parts(krows)
    vc, vs, vl = ref.parts(vrows)
    x = scale * ((kl + ks * kc) @ q)
    p, v = torch.softmax(x, 0), vl + vs * vc
    out = p @ v
    if kept is not None:
        w = torch.exp(x - x.max())[:, None]
        return (cut(w * vs, kept) * vc + w * vl).sum(0) / w.sum()
    # a score: products of codes and queries are exact; a group's, in up to three parts, and its queries are summed in additions that
    # may cut (two half steps; those of zero are exact); then the pair's fused product, up to four groups, the scale and the base-2
    # exponent, from which the largest is taken and whose result is off by a step
    terms = int((q.view(-1, 32) != 0).sum(1).max())
    es = 2 * U * (3 * terms + 16) * (abs(scale) * ((ks * kc + kl.abs()) @ q.abs())) + U * (4 * x.abs() + 4 * x.abs().max() + 8)
    # weights that are off by e_j take the output along by p_j e_j (v_j - out); their products with scales are rounded once and kept to
    # 16 or 24 bits; a wave's sums: in its tiles of 32 tokens (every fourth) up to four products and two fused additions a token, two
    # roundings from one tile to the next; then the lowest values' sum, the quotient, where there are more tokens than a tile's four waves, two
    # roundings each, and a piece every 128 tokens; what adds zero or takes times one is exact
    tiles = -(-n // 128)
    additions = 6 * min(n, 32 * tiles) + 2 * (tiles - 1) + 3 + (8 if n > 32 else 0) + (2 * (n // 128 + 1) if n > 128 else 0)
    bound = (p * es) @ (v - out).abs() + (p * (2.0 ** -KEPT[dtype] + 2 * U)) @ (vs * vc)
    bound += 2 * U * additions * (p @ (15 * vs + vl.abs())) + (2 * U * additions + pref.HALF[dtype]) * out.abs()
    return out, 1.01 * bound


def inputs(seed, dtype, B, H, Hkv, d, page, longest, hot):
    """Sequences of up to `longest` tokens, queries of `hot` channels a group.  Values are such that lost bits show: in bf16, whose result's
    rounding goes with the output, of either sign, so that some outputs are small; in fp32, where it is sums that round, of one sign in a
    group, so that either the lowest value is small or the codes are."""
    gen = torch.Generator().manual_seed(seed)
    width = -(-longest // page)
    lens = torch.randint(1, longest + 1, (B,), generator=gen).tolist()
    table = torch.randperm(B * width, generator=gen).view(B, width).to(torch.int32)
    kp = ref.rows(torch.randn(B * width, Hkv, page, d, generator=gen))
    v = torch.randn(B * width, Hkv, page, d, generator=gen)
    vp = ref.rows(v if dtype == "bf16" else v.abs() * (torch.randint(0, 2, (d // 32,), generator=gen) * 2 - 1).repeat_interleave(32))
    q = torch.randn(B, H, d, generator=gen)
    q = (q.view(B, H, d // 32, 32) * (torch.arange(32) < hot)).view(B, H, d).to(ref.TYPES[dtype])
    return q, kp, vp, table, lens


def each(q, kp, vp, table, lens, page, dtype, scale, **kw):
    out = []
    B, H = q.shape[:2]
    for b in range(B):
        at = table[b, torch.arange(lens[b]) // page].long(), torch.arange(lens[b]) % page
        for h in range(H):
            g = h * kp.shape[1] // H
            out.append(one_head(q[b, h].double(), kp[at[0], g, at[1]], vp[at[0], g, at[1]], scale, dtype, **kw))
    if kw:
        return torch.stack(out).view(q.shape)
    return tuple(torch.stack([x[i] for x in out]).view(q.shape) for i in (0, 1))


CASES = [(24, 4, 2, 128, 8, 6, 1), (24, 8, 1, 64, 16, 3, 1), (8, 12, 1, 128, 64, 20, 32)]


@pytest.mark.parametrize("dtype,fewer", [("bf16", 8), ("bf16", 11), ("f32", 16)])
def test_the_bound_sees_fewer_bits(dtype, fewer):
    """A step of the stated precision is within the bound for every case, one of fewer bits is not."""
    seen = 0
    for i, (B, H, Hkv, d, page, longest, hot) in enumerate(CASES):
        args = (*inputs(i, dtype, B, H, Hkv, d, page, longest, hot), page, dtype, 0.5 if hot == 1 else 0.02)
        want, bound = each(*args)
        off = lambda bits: (each(*args, kept=bits).to(ref.TYPES[dtype]).double() - want).abs() > bound
        assert not bool(off(KEPT[dtype]).any())
        seen += int(off(fewer).sum())
    assert seen >= 20


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_decode_keeps_the_stated_bits(dtype, case):
    B, H, Hkv, d, page, longest, hot = CASES[case]
    q, kp, vp, table, lens = inputs(case, dtype, B, H, Hkv, d, page, longest, hot)
    scale = 0.5 if hot == 1 else 0.02
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    gb.gformer_paged_decode_q4(q.cuda(), None, None, out, kp.cuda(), vp.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                               softmax_scale=scale)
    pref.check(out, *each(q, kp, vp, table, lens, page, dtype, scale), dtype)


@gpu
@pytest.mark.parametrize("dtype,B,H,Hkv,d,page,longest", [("bf16", 300, 16, 1, 128, 16, 140), ("bf16", 2, 4, 1, 128, 16, 1500), ("f32", 2, 2, 1, 64, 32, 700)])
def test_and_in_large_or_long_calls(dtype, B, H, Hkv, d, page, longest):
    """Eight query heads of a key head a workgroup, and sequences that are cut."""
    q, kp, vp, table, lens = inputs(B, dtype, B, H, Hkv, d, page, longest, 2)
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    gb.gformer_paged_decode_q4(q.cuda(), None, None, out, kp.cuda(), vp.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                               softmax_scale=0.3)
    some = list(range(0, B, max(1, B // 12)))
    want, bound = each(q[some], kp, vp, table[some], [lens[b] for b in some], page, dtype, 0.3)
    pref.check(out[some], want, bound, dtype)
