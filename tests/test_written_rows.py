"""Rows that a call writes are different memory: strides that lay two of them over each other are refused, any others are taken."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2412_19829_amd import binding as gb
from paper_2412_19829_amd.rotary import rotary_frequencies
from tests import q4_reference as ref

gpu = pytest.mark.gpu
A = 1 << 20


def params(make, **kw):
    p = make()
    for name, val in kw.items():
        setattr(p, name, (ctypes.c_int64 * 2)(*val))
    return p


# (row, head) strides for d = 64 that lay rows over each other
OVERLAP = [((64, 64), 5, 2),          # row r's head 1 is row r + 1's head 0
           ((128, 160), 4, 2),        # half of a row
           ((192, 384), 3, 2),        # two rows on
           ((64, 128), 3, 2), ((320, 64), 2, 7), ((72, 64), 2, 2), ((1024, 1032), 2, 2), ((1 << 20, 1 << 20), 2, 2)]


def read(strides, rows, heads, name="k_stride"):
    p = params(gb.make_paged_params, **{name: strides})
    return gb.lib().gformer_paged_read_q4(*(i * A for i in range(1, 8)), 2, rows, heads, 64, 9, 4, ctypes.byref(p), None)


# all of these are refused before a device is asked for
@pytest.mark.parametrize("strides,rows,heads", OVERLAP)
def test_read_refuses(strides, rows, heads):
    assert read(strides, rows, heads) == read(strides, rows, heads, "v_stride") == gb.GF_ERR_INVALID_ARG


@pytest.mark.parametrize("strides,rows,heads", OVERLAP)
def test_decode_refuses(strides, rows, heads):
    p = params(gb.make_paged_params, o_stride=strides)
    at = [i * A for i in range(1, 9)]
    assert gb.lib().gformer_paged_decode_q4(*at, rows, heads, 1, 64, 9, 4, 0, ctypes.byref(p), 9 * A, 1 << 30, None) == gb.GF_ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["q_out_stride", "k_out_stride"])
@pytest.mark.parametrize("strides,rows,heads", OVERLAP)
def test_rotary_refuses(strides, rows, heads, name):
    p = params(gb.make_rotary_params, **{name: strides})
    at = [i * A for i in range(1, 6)]
    assert gb.lib().gformer_rotary(*at, 6 * A, 0, 0, 0, rows, heads, heads, 64, ctypes.byref(p), None) == gb.GF_ERR_INVALID_ARG


def test_overlap_is_found_wherever_it_is():
    """Against all pairs of rows, for strides in eights of a row.  Calls of no rows at all are fine, whatever the strides."""
    assert read((64, 64), 0, 2) == gb.GF_OK
    for rows in (2, 3, 6):
        for heads in (2, 3, 5):
            for a in range(64, 64 * 8, 24):
                for b in range(64, 64 * 8, 24):
                    at = sorted(r * a + h * b for r in range(rows) for h in range(heads))
                    if any(y - x < 64 for x, y in zip(at, at[1:])):
                        assert read((a, b), rows, heads) == gb.GF_ERR_INVALID_ARG, (rows, heads, a, b)


@gpu
@pytest.mark.parametrize("strides,rows,heads", [((64, 320), 5, 2), ((128, 192), 4, 2), ((192, 448), 5, 2), ((192, 64), 5, 3), ((72, 4096), 6, 3), ((448, 192), 2, 5), ((64, 64), 1, 3),
                                                ((64, 64), 3, 1)])
def test_rows_apart_in_any_order_are_written(strides, rows, heads):
    gen = torch.Generator().manual_seed(rows)
    lay = lambda: torch.full((rows * strides[0] + heads * strides[1] + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    view = lambda t: t.as_strided((rows, heads, 64), (*strides, 1))
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    x = torch.randn(rows, heads, 64, generator=gen).bfloat16()
    pages = [torch.zeros(2, heads, 8, 40, dtype=torch.uint8, device="cuda") for _ in range(2)]
    table, zero, cu = ints(1).view(1, 1), ints(0), ints(0, rows)
    gb.gformer_paged_fill_q4(x.cuda(), x.cuda(), *pages, table, zero, cu)
    k, v = lay(), lay()
    gb.gformer_paged_read_q4(*pages, view(k), view(v), table, zero, cu)
    held = ref.values(ref.rows(x)).to(torch.bfloat16)
    for t in (k, v):
        assert torch.equal(view(t).cpu(), held) and int((t == 7.0).sum()) >= t.numel() - held.numel()
    q, out, want = lay(), lay(), torch.empty(rows, heads, 64, dtype=torch.bfloat16, device="cuda")
    view(q).copy_(x)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    gb.gformer_rotary(x.cuda(), None, want, None, rotary_frequencies(64), positions=pos)
    gb.gformer_rotary(view(q), None, view(out), None, rotary_frequencies(64), positions=pos)
    gb.gformer_rotary(view(q), None, view(q), None, rotary_frequencies(64), positions=pos)
    assert torch.equal(view(out), want) and torch.equal(view(q), want)
    one, many = lay(), torch.empty(rows, heads, 64, dtype=torch.bfloat16, device="cuda")
    users = (table.expand(rows, 1).contiguous(), torch.full((rows,), rows, dtype=torch.int32, device="cuda"))
    gb.gformer_paged_decode_q4(x.cuda(), None, None, view(one), *pages, *users)
    gb.gformer_paged_decode_q4(x.cuda(), None, None, many, *pages, *users)
    assert torch.equal(view(one), many)
