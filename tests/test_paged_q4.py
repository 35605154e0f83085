"""The paged cache of 4 bits a value: rows into it and out of it, copies of its pages, one new token over it."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

from paper_2412_19829_amd import binding as gb
from paper_2412_19829_amd.paged import PagedCache
from tests import packed_reference as pref
from tests import q4_reference as ref

gpu = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
A = 1 << 20


# ---- refusals (CPU) --------------------------------------------------------------------------------

def wrong(**kw):
    p = gb.make_paged_params()
    for name, val in kw.items():
        setattr(p, name, val if not isinstance(val, tuple) else (ctypes.c_int64 * len(val))(*val))
    return p


def decode(p=None, q=A, k=2 * A, v=3 * A, out=4 * A, kp=5 * A, vp=6 * A, table=7 * A, lens=8 * A, B=2, H=4, Hkv=2, d=64, pages=9,
           width=4, max_len=0, ws=9 * A, ws_bytes=1 << 30):
    p = p or gb.make_paged_params()
    return gb.lib().gformer_paged_decode_q4(q, k, v, out, kp, vp, table, lens, B, H, Hkv, d, pages, width, max_len, ctypes.byref(p), ws,
                                            ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), 1), (dict(k=0), 1), (dict(v=0), 1), (dict(lens=0), 1), (dict(table=0), 1), (dict(kp=0), 1), (dict(out=A), 1),
    (dict(out=5 * A), 1), (dict(vp=5 * A), 1), (dict(q=A + 8), 1), (dict(kp=A + 8), 1), (dict(lens=A + 1), 1), (dict(B=-1), 1), (dict(H=5), 1),
    (dict(Hkv=0), 1), (dict(d=32), 2), (dict(pages=0), 1), (dict(pages=-1), 1), (dict(width=-1), 1), (dict(max_len=-1), 1),
    (dict(width=1 << 25), 2), (dict(p=wrong(page_size=4)), 2), (dict(p=wrong(page_size=0)), 1), (dict(p=wrong(page_size=48)), 2),
    (dict(p=wrong(struct_size=4)), 1), (dict(p=wrong(dtype=7)), 1), (dict(p=wrong(softmax_scale=NAN)), 1),
    (dict(p=wrong(q_stride=(60, 64))), 1), (dict(p=wrong(kpage_stride=(8192, 4096, 32))), 1),     # rows would overlap
    (dict(p=wrong(kpage_stride=(8192, 4096, 44))), 1), (dict(p=wrong(vpage_stride=(8192, -64, 40))), 1),
    (dict(d=128, p=wrong(kpage_stride=(8192, 4096, 88))), 1), (dict(p=wrong(vpage_stride=(1 << 23, 1 << 22, (1 << 20) + 8))), 2),
    (dict(width=64, ws=0), 3), (dict(width=64, ws_bytes=255), 3), (dict(width=64, ws=A + 16), 1), (dict(B=1 << 30, H=4), 2),
])
def test_decode_refusals(kw, status):
    assert decode(**kw) == status


def test_row_calls_and_copy_refusals():
    p, ptrs = gb.make_paged_params(), [i * A for i in range(1, 8)]
    for entry in (gb.lib().gformer_paged_fill_q4, gb.lib().gformer_paged_read_q4):
        call = lambda *a, p=p: entry(*a, ctypes.byref(p), None)
        assert call(*ptrs, 2, 0, 2, 64, 9, 4) == gb.GF_OK and call(*ptrs, 0, 5, 2, 64, 9, 4) == gb.GF_OK
        for i in range(7):
            assert call(*(0 if i == j else x for j, x in enumerate(ptrs)), 2, 5, 2, 64, 9, 4) == gb.GF_ERR_INVALID_ARG
            assert call(*(x + 2 if i == j else x for j, x in enumerate(ptrs)), 2, 5, 2, 64, 9, 4) == gb.GF_ERR_INVALID_ARG
        assert call(*ptrs, -1, 5, 2, 64, 9, 4) == call(*ptrs, 2, -5, 2, 64, 9, 4) == gb.GF_ERR_INVALID_ARG
        assert call(*ptrs, 2, 5, 2, 64, 9, 4, p=wrong(page_size=12)) == call(*ptrs, 2, 5, 2, 96, 9, 4) == gb.GF_ERR_UNSUPPORTED
        assert call(*ptrs, 2, (1 << 30) + 1, 2, 64, 9, 4) == call(*ptrs, 2, 1 << 30, 64, 64, 9, 4) == gb.GF_ERR_UNSUPPORTED
        assert call(*ptrs, 2, 5, 2, 64, 9, 4, p=wrong(k_stride=(64, 64))) != gb.GF_ERR_UNSUPPORTED
    same = lambda i, j: [ptrs[i] if n == j else x for n, x in enumerate(ptrs)]
    assert gb.lib().gformer_paged_fill_q4(*same(2, 3), 2, 5, 2, 64, 9, 4, ctypes.byref(p), None) == gb.GF_ERR_INVALID_ARG
    for i, j in ((0, 2), (0, 3), (1, 2), (2, 3)):      # the rows that are written are nothing else's
        assert gb.lib().gformer_paged_read_q4(*same(i, j), 2, 5, 2, 64, 9, 4, ctypes.byref(p), None) == gb.GF_ERR_INVALID_ARG
    copy = lambda *a, p=p: gb.lib().gformer_pages_copy_q4(*a, ctypes.byref(p), None)
    assert copy(A, 2 * A, 3 * A, 4 * A, 0, 2, 64, 9) == gb.GF_OK
    assert copy(0, 2 * A, 3 * A, 4 * A, 1, 2, 64, 9) == copy(A, A, 3 * A, 4 * A, 1, 2, 64, 9) == gb.GF_ERR_INVALID_ARG
    assert copy(A, 2 * A, 3 * A, 4 * A, -1, 2, 64, 9) == copy(A, 2 * A, 3 * A, 0, 1, 2, 64, 9) == gb.GF_ERR_INVALID_ARG
    assert copy(A, 2 * A, 3 * A, 4 * A, 1, 2, 80, 9) == copy(A, 2 * A, 3 * A, 4 * A, 1 << 30, 2, 64, 9) == gb.GF_ERR_UNSUPPORTED


def test_workspace_is_what_the_chunks_take():
    b = gb.gformer_paged_decode_q4_workspace_bytes
    assert b(1, 4, 2, 64, 100) == 0 and b(1, 4, 3, 64, 1 << 15) == 0 and b(0, 4, 2, 64, 1 << 15) == 0
    need = b(1, 32, 8, 128, 1 << 15)
    assert need % 256 == 0 and need >= 2 * 32 * 130 * 4
    assert b(1, 32, 8, 128, 0, table_width=1 << 9) == need
    for B, H, Hkv, d in ((1, 1, 1, 64), (3, 64, 1, 128), (4096, 32, 8, 64)):    # the longest a table holds, within 32 bits
        assert b(B, H, Hkv, d, 1 << 30) >= 0


def test_binding_refuses():
    z = lambda *s, **kw: torch.zeros(*s, **kw)
    i32 = dict(dtype=torch.int32)
    q, pages = z(2, 4, 64), z(3, 2, 8, 40, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device"):
        gb.gformer_paged_decode_q4(q, None, None, z(2, 4, 64), pages, pages.clone(), z(2, 3, **i32), z(2, **i32))
    with pytest.raises(ValueError, match="device"):
        gb.gformer_paged_fill_q4(z(5, 2, 64), z(5, 2, 64), pages, pages.clone(), z(1, 3, **i32), z(1, **i32), z(2, **i32))
    with pytest.raises(ValueError, match="uint8"):
        gb.gformer_pages_copy_q4(pages, pages.clone(), z(1, **i32), z(1, **i32))


def test_reference_rows_are_within_half_a_scale():
    gen = torch.Generator().manual_seed(3)
    for x in (torch.randn(50, 64, generator=gen), torch.randn(50, 64, generator=gen) * 1e30, torch.randn(50, 64, generator=gen) + 1000):
        codes, scale, low = ref.quantise(x)
        got = ref.values(ref.rows(x))
        step = torch.from_numpy(scale).repeat_interleave(32, -1)
        assert bool(((got - x.double()).abs() <= step / 2 * (1 + 1e-12)).all())


def test_cache_of_4_bits(monkeypatch):
    pairs = []
    monkeypatch.setattr(gb, "gformer_pages_copy_q4", lambda k, v, src, dst: pairs.append((src.tolist(), dst.tolist())))
    c = PagedCache(n_pages=12, page_size=8, n_heads=2, d=128, max_seqs=4, max_pages=5, layers=3, device="cpu", bits=4)
    assert c.kpages.shape == (12, 6, 8, 80) and c.vpages.dtype == torch.uint8 and c.layer(2)[1].shape == (12, 2, 8, 80)
    a = c.open(20)
    c.fork(a)
    assert pairs == [([2], [3])]
    with pytest.raises(ValueError, match="bits"):
        PagedCache(n_pages=12, page_size=8, n_heads=2, d=128, max_seqs=4, max_pages=5, device="cpu", bits=8)


# ---- rows into the cache and out of it (GPU) -------------------------------------------------------

def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def noise(gen, *shape):
    return torch.randint(0, 256, shape, dtype=torch.uint8, generator=gen).cuda()


def same_bytes(got, want, what):
    bad = (got.cpu() != want).nonzero()
    assert not len(bad), f"{what}: {len(bad)} bytes differ, first at {bad[:6].tolist()}: {[(int(got[tuple(i)]), int(want[tuple(i)])) for i in bad[:6]]}"


def special(gen, rows, heads, d, dtype):
    """Groups that are hard to round: ties, constants, one value far away, large offsets, subnormal and huge steps, no numbers."""
    x = torch.randn(rows, heads, d, generator=gen)
    g = x.view(-1, 32)
    kinds = [lambda y: y, lambda y: torch.full_like(y, 0.3), lambda y: torch.zeros_like(y), lambda y: y * 1e-40, lambda y: y * 1e-44,
             lambda y: y * 1e36, lambda y: y + 1e4, lambda y: torch.where(torch.arange(32) == 7, 1e5, y), lambda y: -y.abs(),
             lambda y: torch.arange(32) * 0.5, lambda y: torch.arange(32).clamp(max=30) * 0.25 - 3, lambda y: torch.where(torch.arange(32) == 3, INF, y),
             lambda y: torch.where(torch.arange(32) == 31, NAN, y), lambda y: torch.where(torch.arange(32) == 0, -INF, y),
             lambda y: torch.where(torch.arange(32) == 5, 2.0 ** 127, y), lambda y: torch.where(torch.arange(32) == 5, -1.69e38, y.abs() * 5e37),
             lambda y: -torch.zeros_like(y), lambda y: torch.where(torch.arange(32) == 9, -1e30, 1e-30), lambda y: torch.sign(y) * 1e-45]
    for i in range(g.shape[0]):
        g[i] = kinds[i % len(kinds)](g[i])
    return x.to(dtype)


def expected_fill(pages, x, table, start, lens, page):
    """The cache after rows x went in (CPU)."""
    out, rows, at = pages.cpu().clone(), ref.rows(x), 0
    for s, n in enumerate(lens):
        for i in range(n):
            pos = start[s] + i
            if 0 <= pos < table.shape[1] * page and 0 <= int(table[s, pos // page]) < out.shape[0]:
                out[int(table[s, pos // page]), :, pos % page] = rows[at + i]
        at += n
    return out


def spread(t, wide):
    """The same values as a slice of a wider tensor."""
    if not wide:
        return t
    big = torch.zeros(t.shape[0], t.shape[1] + 3, t.shape[2], dtype=t.dtype, device=t.device)
    big[:, 1:1 + t.shape[1]] = t
    return big[:, 1:1 + t.shape[1]]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page,wide,Hkv", [(64, 8, False, 3), (128, 16, True, 4), (64, 64, True, 8), (128, 8, False, 1)])
def test_fill_and_read(dtype, d, page, wide, Hkv):
    gen = torch.Generator().manual_seed(d + page)
    T = ref.TYPES[dtype]
    lens, start, width, pages = [37, 0, 1, 50, 20], [3, 5, 7, -4, 0], 7, 40
    total = sum(lens) + 6
    k, v = special(gen, total, Hkv, d, T), special(gen, total, Hkv, d, T).flip(0).contiguous()
    table = torch.randperm(pages, generator=gen)[:5 * width].view(5, width).to(torch.int32)
    table[0, 1], table[3, 2], table[4, 0] = -1, pages, 2 ** 31 - 1        # no pages
    row = d * 5 // 8
    shape = (pages, Hkv + 2, page, row)
    kbig, vbig = noise(gen, *shape), noise(gen, *shape)
    kp, vp = kbig[:, 1:1 + Hkv], vbig[:, 1:1 + Hkv]                       # one layer of several
    before = kbig.clone(), vbig.clone()
    want = [expected_fill(p, x, table, start, lens, page) for p, x in ((kp, k), (vp, v))]
    cu = ints(*pref.offsets(lens))
    kd, vd = spread(k.cuda(), wide), spread(v.cuda(), wide)
    gb.gformer_paged_fill_q4(kd, vd, kp, vp, table.cuda(), ints(*start), cu)
    for big, old, w in ((kbig, before[0], want[0]), (vbig, before[1], want[1])):
        old = old.cpu()
        old[:, 1:1 + Hkv] = w
        same_bytes(big, old, "cache")
    # and out again, into rows that hold something
    ko, vo = (spread(torch.full((total, Hkv, d), 7.0, dtype=T, device="cuda"), wide) for _ in range(2))
    gb.gformer_paged_read_q4(kp, vp, ko, vo, table.cuda(), ints(*start), cu)
    for got, pages_ in ((ko, want[0]), (vo, want[1])):
        exp = torch.full((total, Hkv, d), 7.0, dtype=torch.float64)
        held, at = ref.values(pages_), 0
        for s, n in enumerate(lens):
            for i in range(n):
                pos = start[s] + i
                ok = 0 <= pos < width * page and 0 <= int(table[s, pos // page]) < pages
                exp[at + i] = held[int(table[s, pos // page]), :, pos % page] if ok else 0.0
            at += n
        assert torch.equal(torch.nan_to_num(got.cpu().float(), 1e9), torch.nan_to_num(exp.float().to(T).float(), 1e9))


@gpu
@pytest.mark.parametrize("n_seqs", [1, 62, 63, 64, 65, 200])
def test_rows_of_many_sequences(n_seqs):
    """One to three rows of each, some of none, a batch padded behind them."""
    gen = torch.Generator().manual_seed(n_seqs)
    lens = torch.randint(0, 4, (n_seqs,), generator=gen).tolist()
    lens[0] = 3
    start = torch.randint(0, 30, (n_seqs,), generator=gen).tolist()
    total, Hkv, d, page = sum(lens) + 5, 2, 64, 8
    table = torch.randperm(5 * n_seqs, generator=gen).view(n_seqs, 5).to(torch.int32)
    k, v = torch.randn(total, Hkv, d, generator=gen), torch.randn(total, Hkv, d, generator=gen)
    kp, vp = noise(gen, 5 * n_seqs, Hkv, page, 40), noise(gen, 5 * n_seqs, Hkv, page, 40)
    want = [expected_fill(p, x, table, start, lens, page) for p, x in ((kp, k), (vp, v))]
    cu = ints(*pref.offsets(lens))
    gb.gformer_paged_fill_q4(k.cuda(), v.cuda(), kp, vp, table.cuda(), ints(*start), cu)
    same_bytes(kp, want[0], "keys")
    same_bytes(vp, want[1], "values")
    ko, vo = torch.full((total, Hkv, d), 7.0, device="cuda"), torch.full((total, Hkv, d), 7.0, device="cuda")
    gb.gformer_paged_read_q4(kp, vp, ko, vo, table.cuda(), ints(*start), cu)
    for got, x in ((ko, k), (vo, v)):
        assert torch.equal(got[:sum(lens)].cpu(), ref.values(ref.rows(x[:sum(lens)])).float()) and bool((got[sum(lens):] == 7.0).all())


@gpu
def test_fill_rounds_to_even_between_codes():
    # low 0, scale 1: values half way between codes
    x = torch.zeros(1, 1, 64)
    x[0, 0, :15] = torch.arange(15) + 0.5
    x[0, 0, 15] = 15.0
    x[0, 0, 32:47] = -(torch.arange(15) + 0.5)
    x[0, 0, 47] = -15.0
    pages = torch.zeros(2, 1, 1, 8, 40, dtype=torch.uint8, device="cuda")
    for T in (torch.bfloat16, torch.float32):
        gb.gformer_paged_fill_q4(x.to(T).cuda(), x.to(T).cuda(), pages[0], pages[1], ints(0).view(1, 1), ints(2), ints(0, 1))
        codes, scale, low = ref.parts(pages[0, 0, 0, 2])
        assert codes[:16].tolist() == [0, 2, 2, 4, 4, 6, 6, 8, 8, 10, 10, 12, 12, 14, 14, 15]
        assert (scale[0], low[0], scale[32], low[32]) == (1.0, 0.0, 1.0, -15.0)


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_copy(d):
    gen = torch.Generator().manual_seed(d)
    big = [noise(gen, 12, 5, 16, d * 5 // 8) for _ in range(2)]
    pages = [x[:, 1:4] for x in big]
    want = [x.cpu().clone() for x in big]
    src, dst = [0, 3, 7, 5, 20, 2], [9, 1, 7, -1, 4, 11]
    for w in want:
        for i, o in zip(src, dst):
            if i < 12 and 0 <= o < 12:
                w[o, 1:4] = w[i, 1:4]
    gb.gformer_pages_copy_q4(*pages, ints(*src), ints(*dst))
    assert all(torch.equal(x.cpu(), w) for x, w in zip(big, want))


# ---- the decode step (GPU) -------------------------------------------------------------------------

def sound_pages(gen, n, Hkv, page, d):
    return ref.rows(torch.randn(n, Hkv, page, d, generator=gen)).cuda()


def step(gen, dtype, H, Hkv, d, page, lens, *, width=None, new=True, max_len=0, spoil=True, missing=(), scale=None, wide=False):
    """A call over a cache in which everything that is not seen is noise (or no number)."""
    T, B = ref.TYPES[dtype], len(lens)
    own = 1 if new else 0
    width = width or max(1, -(-max(max(lens) + own, 1) // page))
    pages = B * width + 3
    kp, vp = sound_pages(gen, pages, Hkv, page, d), sound_pages(gen, pages, Hkv, page, d)
    table = torch.randperm(pages, generator=gen)[:B * width].view(B, width).to(torch.int32)
    for b, i in missing:
        table[b, i] = -1
    if spoil:
        seen = torch.zeros(pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            for t in range(max(n, 0)):
                if table[b, t // page] >= 0:
                    seen[table[b, t // page], t % page] = True
        for p in (kp, vp):
            bad = torch.full(p.shape, 255, dtype=torch.uint8)             # scales and lowest values that are no number
            p.copy_(torch.where(seen[:, None, :, None], p.cpu(), bad))
    q = spread(torch.randn(B, H, d, generator=gen).to(T).cuda(), wide)
    k, v = (spread(torch.randn(B, Hkv, d, generator=gen).to(T).cuda(), wide) if new else None for _ in range(2))
    out = spread(torch.full((B, H, d), 7.0, dtype=T, device="cuda"), wide)
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    room = min(width * page, max_len or width * page)
    sees = [None if n < 0 or n > room - own else n + own for n in lens]
    # where the new rows go
    kw, vw, lone = kp.cpu().clone(), vp.cpu().clone(), {}
    for b, n in enumerate(lens):
        if new and sees[b] is not None:
            rows = ref.rows(k[b]), ref.rows(v[b])
            if table[b, n // page] < 0:
                lone[b] = rows
            else:
                kw[table[b, n // page], :, n % page], vw[table[b, n // page], :, n % page] = rows
    call = lambda: gb.gformer_paged_decode_q4(q, k, v, out, kp, vp, table.cuda(), ints(*lens), max_len=max_len, softmax_scale=scale)
    return call, q, out, kp, vp, kw, vw, table, sees, scale, room, lone


def check_step(dtype, page, call, q, out, kp, vp, kw, vw, table, sees, scale, room, lone):
    call()
    same_bytes(kp, kw, "keys")
    same_bytes(vp, vw, "values")
    want, bound = ref.decode(q, kw, vw, table, sees, page, scale, dtype, room, lone)
    pref.check(out, want, bound, "out")


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,d,page,lens", [
    (1, 1, 64, 8, [0]), (1, 1, 128, 8, [1]), (4, 4, 64, 16, [15, 16, 17, 0, 31, 32, 33]), (12, 12, 64, 16, [200, 3]),
    (8, 2, 128, 64, [63, 64, 65, 127, 128, 129, 1]), (32, 8, 128, 16, [300, -1, 7]), (8, 1, 128, 32, [100, 31]), (16, 1, 64, 8, [77]),
    (16, 1, 128, 128, [500, 130]), (6, 2, 64, 8, [40, 5]), (6, 2, 128, 8, [40, 5]), (20, 1, 64, 16, [70]), (36, 2, 128, 16, [70]),
])
def test_decode(dtype, H, Hkv, d, page, lens):
    gen = torch.Generator().manual_seed(H * 1000 + d + sum(lens))
    check_step(dtype, page, *step(gen, dtype, H, Hkv, d, page, lens))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [
    dict(lens=[40, 9, -1, 0], new=False), dict(lens=[39, 40, 41, -5], max_len=41), dict(lens=[47, 48, 30], width=6),   # 48: no room
    dict(lens=[100, 64], missing=[(0, 3), (1, 0), (1, 8)]),                # holes, one of them where the new row would go
    dict(lens=[5, 3], missing=[(0, 0), (1, 0)], new=False),               # rows that see nothing
    dict(lens=[70, 20], wide=True), dict(lens=[70, 20], scale=0.0), dict(lens=[70, 20], scale=-3.0), dict(lens=[33, 2], scale=20.0),
])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_rows(dtype, kw, d):
    gen = torch.Generator().manual_seed(len(str(kw)) + d)
    check_step(dtype, 8, *step(gen, dtype, 8, 2, d, 8, **kw))


@gpu
@pytest.mark.parametrize("dtype,H,Hkv,d,page,lens", [
    ("bf16", 8, 2, 128, 64, [2500, 1000, 257]), ("f32", 8, 2, 64, 32, [1500, 3]), ("bf16", 12, 12, 64, 16, [1023]), ("f32", 4, 4, 128, 128, [900]),
])
def test_decode_cut_along_its_length(dtype, H, Hkv, d, page, lens):
    gen = torch.Generator().manual_seed(sum(lens))
    assert gb.gformer_paged_decode_q4_workspace_bytes(len(lens), H, Hkv, d, max(lens) + 1) > 0
    args = step(gen, dtype, H, Hkv, d, page, lens)
    check_step(dtype, page, *args)
    first = args[2].clone()
    args[0]()
    assert torch.equal(first, args[2])                                    # equal calls, equal bits


@gpu
@pytest.mark.parametrize("H,Hkv,page,lens,many", [(16, 2, 16, [700, 3, 129], 200), (12, 1, 8, [300, -1, 500], 300), (40, 4, 64, [200, 90], 100), (5, 1, 16, [260], 700)])
def test_decode_of_two_sets_of_query_heads(H, Hkv, page, lens, many):
    """Calls large enough that a workgroup takes eight query heads: long ones among single tokens."""
    gen = torch.Generator().manual_seed(H)
    lens = lens + torch.randint(0, 2, (many,), generator=gen).tolist()
    args = step(gen, "bf16", H, Hkv, 128, page, lens)
    check_step("bf16", page, *args)
    first = args[2].clone()
    args[0]()
    assert torch.equal(first, args[2])


@gpu
@pytest.mark.parametrize("H,d,lens", [(520, 64, [300]), (400, 128, [129, 140])])
def test_decode_of_so_many_heads_that_nothing_is_cut(H, d, lens):
    gen = torch.Generator().manual_seed(H)
    assert gb.gformer_paged_decode_q4_workspace_bytes(len(lens), H, H, d, max(lens) + 1) == 0
    check_step("bf16", 16, *step(gen, "bf16", H, H, d, 16, lens))


@gpu
@pytest.mark.parametrize("B,H,Hkv,d,most", [(64, 4, 4, 64, 40), (65, 2, 1, 128, 300), (150, 8, 8, 64, 20), (333, 1, 1, 64, 700), (700, 2, 2, 128, 12)])
def test_decode_of_many_sequences(B, H, Hkv, d, most):
    """Shares of the work that hold several sequences, and sequences that lie in several shares, idle ones among them."""
    gen = torch.Generator().manual_seed(B)
    lens = torch.randint(-2, most, (B,), generator=gen).tolist()
    lens[B // 2] = 8 * most
    check_step("bf16", 16, *step(gen, "bf16", H, Hkv, d, 16, lens))


@gpu
def test_decode_keeps_large_offsets_of_values_and_keys():
    # groups whose values lie far from zero, close together
    gen = torch.Generator().manual_seed(8)
    B, H, Hkv, d, page, n = 1, 8, 2, 128, 16, 90
    x = torch.randn(8, Hkv, page, d, generator=gen) * 0.1 + torch.randint(-20, 20, (8, Hkv, page, d // 32), generator=gen).repeat_interleave(32, -1)
    kp, vp = ref.rows(x).cuda(), ref.rows(x.flip(0)).cuda()
    q = torch.randn(B, H, d, generator=gen)
    table = torch.arange(8, dtype=torch.int32).view(1, 8)
    for dtype in ("bf16", "f32"):
        qd = q.to(ref.TYPES[dtype]).cuda()
        out = gb.gformer_paged_decode_q4(qd, None, None, torch.empty_like(qd), kp, vp, table.cuda(), ints(n), softmax_scale=0.02)
        want, bound = ref.decode(qd, kp, vp, table, [n], page, 0.02, dtype, 128)
        pref.check(out, want, bound, dtype)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_no_number_stays_where_it_is_seen(dtype):
    gen = torch.Generator().manual_seed(9)
    T, d, page = ref.TYPES[dtype], 128, 8
    kp, vp = sound_pages(gen, 12, 2, page, d), sound_pages(gen, 12, 2, page, d)
    table = torch.arange(12, dtype=torch.int32).view(3, 4)
    vp[1, 1, 2, d // 2 + 4:d // 2 + 8] = 255           # row 0, token 10, head 1: the second group of its value
    kp[5, 0, 1, d // 2:d // 2 + 4] = 255               # row 1, token 9, head 0: a key
    q = torch.randn(3, 8, d, generator=gen).to(T).cuda()
    out = gb.gformer_paged_decode_q4(q, None, None, torch.zeros_like(q), kp, vp, table.cuda(), ints(20, 20, 20))
    nan = torch.isnan(out).cpu()
    want = torch.zeros(3, 8, d, dtype=torch.bool)
    want[0, 4:, 32:64] = True
    want[1, :4] = True
    assert torch.equal(nan, want)
    # and a new token that holds one
    k = torch.randn(3, 2, d, generator=gen).to(T).cuda()
    v = k.clone()
    v[2, 0, 5] = INF
    out = gb.gformer_paged_decode_q4(q, k, v, torch.zeros_like(q), kp, vp, table.cuda(), ints(-1, -1, 3))
    want[:] = False
    want[2, :4, :32] = True
    assert torch.equal(torch.isnan(out).cpu(), want) and bool((out[:2] == 0).all())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_read_of_more_than_the_last_cache_holds(dtype):
    gen = torch.Generator().manual_seed(5)
    T, Hkv, d, page = ref.TYPES[dtype], 16, 128, 64
    n = (300 << 20) // (2 * Hkv * d * (2 if dtype == "bf16" else 4)) + 5
    kp, vp = sound_pages(gen, 3, Hkv, page, d), sound_pages(gen, 3, Hkv, page, d)
    table = torch.randint(0, 3, (1, -(-n // page)), generator=gen).to(torch.int32)
    ko, vo = (torch.zeros(n, Hkv, d, dtype=T, device="cuda") for _ in range(2))
    gb.gformer_paged_read_q4(kp, vp, ko, vo, table.cuda(), ints(0), ints(0, n))
    for got, pages in ((ko, kp), (vo, vp)):
        held = ref.values(pages).float().to(T).cuda().transpose(1, 2)         # [pages, tokens, heads, d]
        want = held[table[0].long().cuda()].flatten(0, 1)[:n]
        assert torch.equal(got, want)


@gpu
def test_far_pages():
    """Pages whose offsets pass 32 bits."""
    gen = torch.Generator().manual_seed(4)
    d, page, Hkv, n = 128, 64, 8, 150
    count = (1 << 32) // (80 * page * Hkv) + 60
    kp, vp = (torch.empty(count, Hkv, page, 80, dtype=torch.uint8, device="cuda") for _ in range(2))
    far = torch.tensor([count - 1, count - 30, count - 2], dtype=torch.int32).view(1, 3)
    k, v = (torch.randn(n, Hkv, d, generator=gen).bfloat16().cuda() for _ in range(2))
    gb.gformer_paged_fill_q4(k, v, kp, vp, far.cuda(), ints(0), ints(0, n))
    gb.gformer_pages_copy_q4(kp, vp, ints(count - 1), ints(count - 3))
    far[0, 0] = count - 3
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    gb.gformer_paged_read_q4(kp, vp, ko, vo, far.cuda(), ints(0), ints(0, n))
    assert torch.equal(ko.cpu(), ref.values(ref.rows(k)).float().bfloat16()) and torch.equal(vo.cpu(), ref.values(ref.rows(v)).float().bfloat16())
    q = torch.randn(1, 16, d, generator=gen).bfloat16().cuda()
    out = gb.gformer_paged_decode_q4(q, None, None, torch.empty_like(q), kp, vp, far.cuda(), ints(n), softmax_scale=0.09)
    rows = ref.rows(k), ref.rows(v)
    for h in (0, 7, 15):
        want, bound = ref.one_head(q[0, h].double().cpu(), rows[0][:, h // 2], rows[1][:, h // 2], 0.09, "bf16")
        pref.check(out[0, h], want, bound, f"head {h}")


@gpu
@pytest.mark.parametrize("quick", [True, False])
def test_a_named_stream_and_the_binding_without_its_module(quick, monkeypatch):
    """Every call on a stream that is named, through the extension module and through the binding's own code."""
    gen = torch.Generator().manual_seed(16)
    H, Hkv, d, page, lens = 8, 2, 64, 16, [700, 30]
    if not quick:
        monkeypatch.setattr(gb, "_quick", lambda *a: False)
    kp, vp = sound_pages(gen, 100, Hkv, page, d), sound_pages(gen, 100, Hkv, page, d)
    kw, vw = kp.cpu().clone(), vp.cpu().clone()
    table = torch.randperm(98, generator=gen)[:92].view(2, 46).to(torch.int32)
    k, v = torch.randn(5, Hkv, d, generator=gen).cuda(), torch.randn(5, Hkv, d, generator=gen).cuda()
    q, out = torch.randn(2, H, d, generator=gen).cuda(), torch.zeros(2, H, d, device="cuda")
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    tab, ln, start, cu = table.cuda(), ints(*lens), ints(698, 28), ints(0, 3, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on = side.cuda_stream
    gb.gformer_paged_fill_q4(k, v, kp, vp, tab, start, cu, stream=on)
    gb.gformer_paged_decode_q4(q, k[:2], v[:2], out, kp, vp, tab, ln, softmax_scale=0.125, stream=on)
    gb.gformer_paged_read_q4(kp, vp, ko, vo, tab, start, cu, stream=on)
    gb.gformer_pages_copy_q4(kp, vp, ints(3), ints(99), stream=on)
    torch.cuda.synchronize()
    kw, vw = (expected_fill(p, x.cpu(), table, [698, 28], [3, 2], page) for p, x in ((kw, k), (vw, v)))
    for b, n in enumerate(lens):     # the step's own tokens, in front of the rows that the fill had put there
        for p, x in ((kw, k), (vw, v)):
            p[table[b, n // page], :, n % page] = ref.rows(x[b])
    want, bound = ref.decode(q, kw, vw, table, [n + 1 for n in lens], page, 0.125, "f32", 46 * page)
    pref.check(out, want, bound, "out")
    for got, p in ((ko, kw), (vo, vw)):
        held = ref.values(p).float()
        rows = [held[table[0, t // page], :, t % page] for t in (698, 699, 700)] + [held[table[1, t // page], :, t % page] for t in (28, 29)]
        assert torch.equal(got.cpu(), torch.stack(rows))
    kw[99], vw[99] = kw[3], vw[3]
    same_bytes(kp, kw, "keys")
    same_bytes(vp, vw, "values")


@gpu
def test_streams_and_graphs():
    """Calls on another stream, and a captured run of fill, step and read that is replayed with new inputs."""
    gen = torch.Generator().manual_seed(6)
    H, Hkv, d, page, B = 8, 2, 128, 16, 3
    kp, vp = (torch.zeros(40, Hkv, page, 80, dtype=torch.uint8, device="cuda") for _ in range(2))
    table = torch.randperm(40, generator=gen)[:36].view(3, 12).to(torch.int32).cuda()
    lens, start, cu = ints(100, 40, 0), ints(90, 38, 0), ints(0, 10, 12, 12)
    kn, vn = (torch.randn(12, Hkv, d, generator=gen).bfloat16().cuda() for _ in range(2))
    q, out = torch.randn(B, H, d, generator=gen).bfloat16().cuda(), torch.zeros(B, H, d, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.randn(B, Hkv, d, generator=gen).bfloat16().cuda() for _ in range(2))
    ko, vo = torch.zeros_like(kn), torch.zeros_like(vn)
    ws = torch.empty(gb.gformer_paged_decode_q4_workspace_bytes(B, H, Hkv, d, 192), dtype=torch.uint8, device="cuda")

    def run():
        gb.gformer_paged_fill_q4(kn, vn, kp, vp, table, start, cu)
        gb.gformer_paged_decode_q4(q, k, v, out, kp, vp, table, lens, workspace=ws, softmax_scale=0.1)
        gb.gformer_paged_read_q4(kp, vp, ko, vo, table, start, cu)

    run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        for t in (kn, vn, q, k, v):
            t.copy_(torch.randn(t.shape, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, kp, vp, ko, vo)]
        for t in (out, ko, vo):
            t.zero_()
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, kp, vp, ko, vo))), i


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_its_continuation_and_steps(dtype):
    """Prompts into a cache of 4 bits, one of them forked, a chunk that goes on behind cached tokens through packed attention, and
    steps of all of them: every step's output against attention in 64 bits over what the cache holds."""
    gen = torch.Generator().manual_seed(12)
    T, H, Hkv, d, page, scale = ref.TYPES[dtype], 8, 2, 64, 8, 0.125
    c = PagedCache(n_pages=64, page_size=page, n_heads=Hkv, d=d, max_seqs=3, max_pages=10, layers=2, bits=4)
    kp, vp = c.layer(1)
    rand = lambda *s: torch.randn(*s, generator=gen).to(T).cuda()
    a = c.open(21)
    k, v = rand(21, Hkv, d), rand(21, Hkv, d)
    row = lambda seqs: (c.table[seqs], ints(*(0 for _ in seqs)))
    gb.gformer_paged_fill_q4(k, v, kp, vp, *row([a]), ints(0, 21))
    b = c.fork(a)
    # five more tokens of b
    c.reserve([b])
    for _ in range(5):
        c.reserve([b])
        c.advance([b])
    k2, v2 = rand(5, Hkv, d), rand(5, Hkv, d)
    gb.gformer_paged_fill_q4(k2, v2, kp, vp, c.table[[b]], ints(21), ints(0, 5))
    ka, va = torch.zeros(26, Hkv, d, dtype=T, device="cuda"), torch.zeros(26, Hkv, d, dtype=T, device="cuda")
    gb.gformer_paged_read_q4(kp, vp, ka, va, *row([b]), ints(0, 26))
    for got, first, then in ((ka, k, k2), (va, v, v2)):
        want = torch.cat([ref.values(ref.rows(first)), ref.values(ref.rows(then))]).float().to(T)
        assert torch.equal(got.cpu(), want)
    q = rand(5, H, d)
    out = gb.gformer_packed_attn_fwd(q, ka, va, torch.zeros_like(q), ints(0, 5), ints(0, 26), softmax_scale=scale)
    want, bound = pref.packed(q, ka, va, None, [5], [26], scale, dtype)["out"]
    pref.check(out, want, bound, "chunk")
    e = c.open(0)
    seqs = [a, b, e]
    assert sorted(seqs) == [0, 1, 2]
    for i in range(10):
        c.reserve(seqs)
        q, k, v = rand(3, H, d), rand(3, Hkv, d), rand(3, Hkv, d)
        lens = [c.length(s) for s in range(3)]
        out = gb.gformer_paged_decode_q4(q, k, v, torch.zeros_like(q), kp, vp, c.table, c.lens, softmax_scale=scale)
        want, bound = ref.decode(q, kp, vp, c.table.cpu(), [n + 1 for n in lens], page, scale, dtype, 80)
        pref.check(out, want, bound, f"step {i}")
        c.advance(seqs)
        if i == 4:
            c.free(a)
            c.compact()
            a = c.open(0)
            seqs = [a, b, e]
