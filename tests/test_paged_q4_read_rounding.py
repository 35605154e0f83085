"""gformer_paged_read_q4 rounds what a code stands for once, also where 32 or 64 bits do not hold it."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2412_19829_amd import binding as gb
from tests import q4_reference as ref

gpu = pytest.mark.gpu


def rounded(codes, scale, low, dtype):
    """l + s n (64 bits, multiples of 2^-140 below 2^60) to 8 or 24 significant bits, half to even, in whole numbers: a sum in 64 bits would
    lose a lowest value 2^53 times below the step, and torch's own way to bf16 goes through 32 bits."""
    def one(x):
        n = abs(x)
        k = n.bit_length() - (8 if dtype == "bf16" else 24)
        if k > 0:
            rest, half = n & ((1 << k) - 1), 1 << (k - 1)
            n = (n >> k) + (rest > half or (rest == half and n >> k & 1)) << k
        return math.ldexp(n if x >= 0 else -n, -140)

    whole = lambda t: [int(x) for x in (t.flatten() * 2.0 ** 140).tolist()]
    x = [one(a + b) for a, b in zip(whole(low), whole(scale * codes))]
    return torch.tensor(x, dtype=torch.float64).view(codes.shape).to(ref.TYPES[dtype])


def test_rounding_of_the_test():
    t = lambda *x: torch.tensor(x, dtype=torch.float64)
    far = 2.0 ** -130
    s, l = t(129 / 128, 129 / 128, 129 / 128, 129 / 128, 1.0, 257 / 256), t(-2.0 ** -30, 0.0, far, -far, -2.0 - 2.0 ** -8 - 2.0 ** -40, -4.0)
    assert rounded(t(3.0, 3.0, 3.0, 3.0, 1.0, 3.0), s, l, "bf16").tolist() == [3.015625, 3.03125, 3.03125, 3.015625, -1.0078125, -0.98828125]
    assert (t(387 / 128) - far).to(torch.bfloat16)[0] == 3.03125


def read(pages, n, dtype):
    """The first n tokens of a page of one head."""
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    out = [torch.full((n, 1, pages.shape[-1] * 8 // 5), 7.0, dtype=ref.TYPES[dtype], device="cuda") for _ in range(2)]
    gb.gformer_paged_read_q4(pages, pages.clone(), *out, ints(0).view(1, 1), ints(0), ints(0, n))
    assert torch.equal(out[0], out[1])
    return out[0].cpu()[:, 0]


def hard_rows(d):
    """Rows of one head: all 128 steps of 8 bits with every code, the lowest value from 2^-6 to 2^-60 steps on either side of zero."""
    page, gen = 4096, torch.Generator().manual_seed(d)
    r = torch.arange(page)
    scale = (1 + (r % 128) / 128) * 2.0 ** (r // 128 % 9 * 13.0 - 50)
    rows = torch.zeros(page, d // 2 + d // 8, dtype=torch.uint8)
    code = torch.stack([torch.cat([torch.randperm(16, generator=gen), torch.randperm(16, generator=gen)]) for _ in range(d // 32)]).flatten()
    rows[:, :d // 2] = (code[0::2] | code[1::2] << 4).to(torch.uint8)
    far = torch.randint(6, 61, (page, d // 32), generator=gen)
    low = scale[:, None] * 2.0 ** -far.double() * (torch.randint(0, 3, far.shape, generator=gen) - 1.0)
    pair = torch.stack([scale[:, None].expand_as(low), low], -1).to(torch.bfloat16)
    rows[:, d // 2:] = pair.contiguous().view(torch.uint8).view(page, -1)
    return rows


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_lowest_value_far_below_the_step(dtype, d):
    """All 128 steps of 8 bits with every code, the lowest value from 2^-6 to 2^-60 steps on either side of zero."""
    rows = hard_rows(d)
    want = rounded(*ref.parts(rows), dtype)
    assert dtype == "f32" or int((want != ref.values(rows).float().to(torch.bfloat16)).sum()) > 1000      # where two roundings differ from one
    assert torch.equal(read(rows.view(1, 1, *rows.shape).cuda(), len(rows), dtype), want)


@gpu
def test_such_rows_past_the_caches():
    """More rows than the last cache holds, which go past it: those are written twice there, too."""
    rows, d = hard_rows(128), 128
    n = (256 << 20) // (2 * d * 2) + 777
    pages = rows.view(4, 1, len(rows) // 4, -1).cuda()
    gen = torch.Generator().manual_seed(3)
    table = torch.randint(0, 4, (1, -(-n // pages.shape[2])), generator=gen).to(torch.int32)
    k, v = (torch.zeros(n, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    gb.gformer_paged_read_q4(pages, pages.clone(), k, v, table.cuda(), ints(0), ints(0, n))
    want = rounded(*ref.parts(rows), "bf16").cuda().view(4, -1, d)[table[0].long().cuda()].flatten(0, 1)[:n]
    assert torch.equal(k[:, 0], want) and torch.equal(v[:, 0], want)


@gpu
def test_such_a_group_as_it_is_written():
    x = torch.full((1, 1, 64), -2.0 ** -30)
    x[0, 0, 1], x[0, 0, 2] = 15.0625, 3.0
    x[0, 0, 32:] = -x[0, 0, :32]
    ints = lambda *y: torch.tensor(y, dtype=torch.int32, device="cuda")
    kp, vp = (torch.zeros(1, 1, 8, 40, dtype=torch.uint8, device="cuda") for _ in range(2))
    gb.gformer_paged_fill_q4(x.bfloat16().cuda(), x.bfloat16().cuda(), kp, vp, ints(0).view(1, 1), ints(0), ints(0, 1))
    codes, scale, low = ref.parts(kp[0, 0, 0])
    assert (codes[2], scale[0], low[0]) == (3.0, 129 / 128, -2.0 ** -30)
    got = read(kp, 1, "bf16")[0]
    assert got[2] == 3.015625 and torch.equal(got, rounded(codes, scale, low, "bf16"))
