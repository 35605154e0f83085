"""The paged cache: one new token over it, what fills and moves its pages, and its bookkeeping."""
from __future__ import annotations

import ctypes
import math
import random

import pytest
import torch

from paper_2412_19829_amd import binding as gb
from paper_2412_19829_amd.paged import PagedCache
from tests import packed_reference as ref

gpu = pytest.mark.gpu
NAN = float("nan")
A = 1 << 20


# ---- refusals and bookkeeping (CPU) ----------------------------------------------------------------

def wrong(**kw):
    p = gb.make_paged_params()
    for name, val in kw.items():
        setattr(p, name, val if not isinstance(val, tuple) else (ctypes.c_int64 * len(val))(*val))
    return p


def decode(p=None, q=A, k=2 * A, v=3 * A, out=4 * A, kp=5 * A, vp=6 * A, table=7 * A, lens=8 * A, B=2, H=4, Hkv=2, d=64, pages=9,
           width=4, max_len=0, ws=9 * A, ws_bytes=1 << 30):
    p = p or gb.make_paged_params()
    return gb.lib().gformer_paged_decode(q, k, v, out, kp, vp, table, lens, B, H, Hkv, d, pages, width, max_len, ctypes.byref(p), ws,
                                         ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), 1), (dict(k=0), 1), (dict(v=0), 1), (dict(lens=0), 1), (dict(table=0), 1), (dict(kp=0), 1), (dict(out=A), 1),
    (dict(out=5 * A), 1), (dict(vp=5 * A), 1), (dict(q=A + 8), 1), (dict(lens=A + 1), 1), (dict(B=-1), 1), (dict(H=5), 1), (dict(Hkv=0), 1),
    (dict(d=32), 2), (dict(pages=0), 1), (dict(pages=-1), 1), (dict(width=-1), 1), (dict(max_len=-1), 1), (dict(width=1 << 25), 2),
    (dict(p=wrong(page_size=4)), 2), (dict(p=wrong(page_size=0)), 1), (dict(p=wrong(page_size=48)), 2), (dict(p=wrong(page_size=1 << 17)), 2),
    (dict(p=wrong(struct_size=4)), 1), (dict(p=wrong(dtype=7)), 1), (dict(p=wrong(softmax_scale=NAN)), 1), (dict(p=wrong(q_stride=(60, 64))), 1),
    (dict(p=wrong(kpage_stride=(8192, 4096, 32))), 1), (dict(p=wrong(vpage_stride=(8192, -64, 64))), 1),
    (dict(width=64, ws=0), 3), (dict(width=64, ws_bytes=255), 3), (dict(width=64, ws=A + 16), 1), (dict(B=1 << 30, H=4), 2),
])
def test_decode_refusals(kw, status):
    assert decode(**kw) == status


def test_fill_and_copy_refusals():
    p = gb.make_paged_params()
    fill = lambda *a, p=p: gb.lib().gformer_paged_fill(*a, ctypes.byref(p), None)
    ptrs = [i * A for i in range(1, 8)]
    assert fill(*ptrs, 2, 0, 2, 64, 9, 4) == gb.GF_OK and fill(*ptrs, 0, 5, 2, 64, 9, 4) == gb.GF_OK
    for i in range(7):
        assert fill(*(0 if i == j else x for j, x in enumerate(ptrs)), 2, 5, 2, 64, 9, 4) == gb.GF_ERR_INVALID_ARG
    assert fill(*ptrs, -1, 5, 2, 64, 9, 4) == fill(*ptrs, 2, -5, 2, 64, 9, 4) == gb.GF_ERR_INVALID_ARG
    assert fill(*ptrs, 2, 5, 2, 64, 9, 4, p=wrong(page_size=12)) == gb.GF_ERR_UNSUPPORTED
    copy = lambda *a, p=p: gb.lib().gformer_pages_copy(*a, ctypes.byref(p), None)
    assert copy(A, 2 * A, 3 * A, 4 * A, 0, 2, 64, 9) == gb.GF_OK
    assert copy(0, 2 * A, 3 * A, 4 * A, 1, 2, 64, 9) == copy(A, A, 3 * A, 4 * A, 1, 2, 64, 9) == gb.GF_ERR_INVALID_ARG
    assert copy(A, 2 * A, 3 * A, 4 * A, -1, 2, 64, 9) == copy(A, 2 * A, 3 * A, 0, 1, 2, 64, 9) == gb.GF_ERR_INVALID_ARG
    assert copy(A, 2 * A, 3 * A, 4 * A, 1, 2, 80, 9) == copy(A, 2 * A, 3 * A, 4 * A, 1 << 30, 2, 64, 9) == gb.GF_ERR_UNSUPPORTED


def test_workspace_is_what_the_chunks_take():
    b = gb.gformer_paged_decode_workspace_bytes
    assert b(1, 4, 2, 64, 100) == 0                     # one chunk: nothing to join
    assert b(1, 4, 3, 64, 1 << 15) == 0                 # refused
    need = b(1, 32, 8, 128, 1 << 15)
    assert need % 256 == 0 and need >= 2 * 32 * 130 * 4
    assert b(1, 32, 8, 128, 0, table_width=1 << 9) == need


class Copies:
    """What the cache would have copied."""
    def __init__(self, monkeypatch):
        self.pairs = []
        monkeypatch.setattr(gb, "gformer_pages_copy", lambda k, v, src, dst: self.pairs.append((src.tolist(), dst.tolist())))


def cache(**kw):
    return PagedCache(**{**dict(n_pages=12, page_size=8, n_heads=2, d=64, max_seqs=4, max_pages=5, device="cpu"), **kw})


def test_bookkeeping(monkeypatch):
    done, c = Copies(monkeypatch), cache()
    a = c.open(20)
    assert c.pages(a) == [0, 1, 2] and c.length(a) == 20 and c.lens.tolist() == [20, -1, -1, -1]
    b = c.fork(a)                                       # two full pages shared, the third copied
    assert c.pages(b) == [0, 1, 3] and done.pairs == [([2], [3])] and c.free_pages == 8
    for _ in range(4):
        c.reserve([a])
        c.advance([a])
    assert c.length(a) == 24 and c.pages(a) == [0, 1, 2]
    d = c.fork(a)                                       # every page full: nothing copied
    assert c.pages(d) == [0, 1, 2] and len(done.pairs) == 1
    c.reserve([a, d, a])
    assert c.pages(a)[3] == 4 and c.pages(d)[3] == 5
    e = c.fork(a)                                       # reserved but not written: not part of the fork
    assert c.pages(e) == [0, 1, 2]
    with pytest.raises(RuntimeError, match="sequences"):
        c.open(1)
    c.free(a)
    assert c.table[a].tolist() == [-1] * 5 and c.lens[a] == -1 and c.free_pages == 7
    c.free(b)
    assert c.free_pages == 8 and sorted(p for p, n in enumerate(c._held) if n) == [0, 1, 2, 5]
    assert c.compact() == 1 and done.pairs[-1] == ([5], [3]) and c.pages(d) == [0, 1, 2, 3]
    assert c.compact() == 0 and c.table[d].tolist() == [0, 1, 2, 3, -1]
    with pytest.raises(ValueError, match="no sequence"):
        c.free(a)
    with pytest.raises(ValueError, match="no slot"):
        c.advance([e])


@pytest.mark.parametrize("kw", [dict(n_pages=0), dict(max_seqs=0), dict(layers=0), dict(d=80), dict(dtype=torch.float16), dict(page_size=4),
                                dict(page_size=24), dict(page_size=1 << 17), dict(page_size=1 << 16, max_pages=(1 << 14) + 1)])
def test_a_cache_that_the_calls_would_refuse_is_not_made(kw):
    with pytest.raises(ValueError):
        cache(**kw)


def test_a_refused_call_changes_nothing(monkeypatch):
    Copies(monkeypatch)
    c = cache(n_pages=4)
    a = c.open(30)
    before = (list(c._held), list(c._free), [list(p or []) for p in c._pages], list(c._len))
    for call in (lambda: c.open(8), lambda: c.fork(a), lambda: c.open(41), lambda: c.open(-1), lambda: c.reserve([a, 3])):
        with pytest.raises((RuntimeError, ValueError)):
            call()
        assert before == (c._held, c._free, [list(p or []) for p in c._pages], c._len)


def test_random_lives(monkeypatch):
    Copies(monkeypatch)
    rng, c, live = random.Random(5), cache(n_pages=20, max_seqs=6), []
    for _ in range(500):
        try:
            what = rng.choice(["open", "fork", "free", "step", "step", "step", "compact"])
            if what == "open":
                live.append(c.open(rng.randint(0, 40)))
            elif what == "fork" and live:
                live.append(c.fork(rng.choice(live)))
            elif what == "free" and live:
                c.free(live.pop(rng.randrange(len(live))))
            elif what == "step" and live:
                some = rng.sample(live, rng.randint(1, len(live)))
                c.reserve(some)
                c.advance(some)
            elif what == "compact":
                c.compact()
                assert sorted(c._free) == list(range(20 - len(c._free), 20))
        except (RuntimeError, ValueError):
            pass
        held = [0] * 20
        for s in live:
            for p in c.pages(s):
                held[p] += 1
            assert len(c.pages(s)) * 8 >= c.length(s)
        assert held == c._held and sorted(c._free) == [p for p, n in enumerate(held) if not n]
        # what a sequence still writes into is its own
        assert all(held[c.pages(s)[c.length(s) // 8]] == 1 for s in live if c.length(s) // 8 < len(c.pages(s)))


# ---- GPU -------------------------------------------------------------------------------------------

def make(lens, H, Hkv, d, page, dtype, seed, new=True, width=None, fill=NAN, layout="heads"):
    """A cache whose pages lie anywhere, with `fill` in every slot that holds no token, and the new token."""
    gen = torch.Generator().manual_seed(seed)
    dt = ref.TYPES[dtype]
    need = [max(1, -(-(x + 1) // page)) for x in lens]
    pages, width = sum(need) + 2, width or max(need)
    order = torch.randperm(pages, generator=gen).tolist()
    shape = (pages, Hkv, page, d) if layout == "heads" else (pages, page, Hkv, d)
    kp, vp = (torch.full(shape, fill, dtype=dt) for _ in range(2))
    if layout != "heads":
        kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    ks, vs = [], []
    for b, n in enumerate(lens):
        own = [order.pop() for _ in range(need[b])]
        table[b, :len(own)] = torch.tensor(own)
        k, v = (torch.randn(max(n, 0), Hkv, d, generator=gen).to(dt) for _ in range(2))
        for t in range(n):
            kp[own[t // page], :, t % page], vp[own[t // page], :, t % page] = k[t], v[t]
        ks.append(k)
        vs.append(v)
    q = torch.randn(len(lens), H, d, generator=gen).to(dt)
    k, v = (torch.randn(len(lens), Hkv, d, generator=gen).to(dt) if new else None for _ in range(2))
    dev = lambda t: None if t is None else t.cuda()
    return dict(q=dev(q), k=dev(k), v=dev(v), kpages=kp.cuda(), vpages=vp.cuda(), table=table.cuda(),
                lens=torch.tensor(lens, dtype=torch.int32).cuda()), ks, vs


def expect(x, ks, vs, scale, dtype):
    """out and its bound, from the sequences' rows."""
    q = x["q"].cpu()
    out, bound = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for b in range(q.shape[0]):
        k, v = ks[b], vs[b]
        if x["k"] is not None and x["lens"][b] >= 0:
            k, v = torch.cat([k, x["k"][b:b + 1].cpu()]), torch.cat([v, x["v"][b:b + 1].cpu()])
        if len(k):
            # numerator and denominator see the same rounded weights, so the bound has the weight's rounding twice
            G = q.shape[1] // k.shape[1]
            for h in range(q.shape[1]):
                kh, vh = k[:, h // G].double(), v[:, h // G].double()
                got = ref.sequence(q[b, h:h + 1].double(), kh, vh, None, scale, dtype)
                p = torch.softmax(scale * (q[b, h].double() @ kh.T), 0)
                out[b, h] = got["out"][0][0]
                bound[b, h] = got["out"][1][0] + ref.HALF[dtype] * (p @ vh.abs()) + 64 * ref.U * (p @ vh.abs())
    return out, bound


def step(x, scale, **kw):
    out = torch.full_like(x["q"], 7.0)
    gb.gformer_paged_decode(x["q"], x["k"], x["v"], out, x["kpages"], x["vpages"], x["table"], x["lens"], softmax_scale=scale, **kw)
    torch.cuda.synchronize()
    return out


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(3, 3), (8, 2), (16, 1), (40, 2)])
@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("new", [True, False])
def test_decode(dtype, d, H, Hkv, page, new):
    lens = [0, 1, 7, 8, 31, 32, 33, 127, 128, 700]
    x, ks, vs = make(lens, H, Hkv, d, page, dtype, H + page, new, layout="heads" if page == 8 else "tokens")
    before = (x["kpages"].clone(), x["vpages"].clone())
    got = step(x, d ** -0.5)
    ref.check(got, *expect(x, ks, vs, d ** -0.5, dtype), "out")
    for pages, old, rows in ((x["kpages"], before[0], x["k"]), (x["vpages"], before[1], x["v"])):
        if new:                                          # the new token's slot, and nothing else
            for b, t in enumerate(lens):
                old[x["table"][b, t // page].long(), :, t % page] = rows[b]
        assert torch.equal(pages.view(torch.int16 if dtype == "bf16" else torch.int32), old.view(torch.int16 if dtype == "bf16" else torch.int32))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
def test_decode_scales(dtype, scale):
    x, ks, vs = make([40, 300], 4, 2, 64, 16, dtype, 3)
    ref.check(step(x, scale), *expect(x, ks, vs, scale, dtype), "out")


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_and_short_sequences_in_one_call(dtype):
    lens = [9000, 3, 2500, 0]
    x, ks, vs = make(lens, 8, 2, 128, 128, dtype, 4)
    want = expect(x, ks, vs, 0.09, dtype)
    ref.check(step(x, 0.09), *want, "bound by the table")
    ref.check(step(x, 0.09, max_len=9001), *want, "bound by max_len")
    # a bound that is too small: the sequence is idle, the others are not
    got = step(x, 0.09, max_len=2501)
    assert (got[0] == 0).all()
    ref.check(got[1:], want[0][1:], want[1][1:], "the others")


@gpu
def test_idle_rows_and_pages_that_are_none():
    lens = [-1, 20, 64, -2147483648, 2147483647, 30]
    x, ks, vs = make([max(0, min(n, 64)) for n in lens], 4, 2, 64, 16, "f32", 5)
    x["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    x["table"] = torch.cat([x["table"][:, :4], torch.full((6, 0), -1, dtype=torch.int32).cuda()], 1).contiguous()
    before = x["kpages"].clone()
    # sequence 2 is full (four pages of 16): no room for a token
    x["table"][5, 0] = 1 << 30                           # the first 16 tokens of sequence 5 are not there
    got = step(x, 0.125)
    for b in (0, 2, 3, 4):
        assert (got[b] == 0).all(), b
    want = expect({**x, "lens": [20, 30], **{n: x[n][[1, 5]] for n in "qkv"}}, [ks[1], ks[5][16:]], [vs[1], vs[5][16:]], 0.125, "f32")
    ref.check(got[[1, 5]], *want, "out")
    changed = (torch.nan_to_num(x["kpages"], 9.0) != torch.nan_to_num(before, 9.0)).any(-1).any(1).nonzero().tolist()
    assert sorted(changed) == sorted([[int(x["table"][1, 1]), 4], [int(x["table"][5, 1]), 14]])
    # the new token's page is none: it is seen, and not written
    x["table"][1, 1] = -5
    before = x["kpages"].clone()
    got = step(x, 0.125)
    want = expect({**x, "lens": [16], **{n: x[n][[1]] for n in "qkv"}}, [ks[1][:16]], [vs[1][:16]], 0.125, "f32")
    ref.check(got[[1]], *want, "out")
    assert torch.equal(torch.nan_to_num(x["kpages"], 9.0), torch.nan_to_num(before, 9.0))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_fill(dtype):
    gen = torch.Generator().manual_seed(1)
    lens, start, page, Hkv, d = [5, 0, 70, 33, 9], [0, 3, 30, -4, 60], 16, 3, 64
    k, v = (torch.randn(sum(lens) + 40, 2 * Hkv, d, generator=gen).to(ref.TYPES[dtype]).cuda()[:, i::2] for i in range(2))
    width, pages = 5, 30
    table = torch.randperm(pages, generator=gen)[:25].view(5, 5).to(torch.int32)
    table[2, 3], table[3, 0] = pages, -1
    kp, vp = (torch.zeros(pages, page, Hkv, d, dtype=k.dtype).cuda().transpose(1, 2) for _ in range(2))
    want = [kp.clone(), vp.clone()]
    at = 0
    for s, n in enumerate(lens):
        for i in range(n):
            t = start[s] + i
            if 0 <= t < width * page and 0 <= table[s, t // page] < pages:
                for w, x in zip(want, (k, v)):
                    w[int(table[s, t // page]), :, t % page] = x[at + i]
        at += n
    gb.gformer_paged_fill(k, v, kp, vp, table.cuda(), torch.tensor(start, dtype=torch.int32).cuda(),
                          torch.tensor(ref.offsets(lens), dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 8), (128, 64), (64, 512)])
def test_copy(dtype, d, page):
    gen = torch.Generator().manual_seed(2)
    kp, vp = (torch.randn(9, 3, page, d, generator=gen).to(ref.TYPES[dtype]).cuda() for _ in range(2))
    vp = vp.transpose(1, 2).contiguous().transpose(1, 2)
    want = [kp.clone(), vp.clone()]
    src, dst = [8, 1, 7, 3, -1, 2], [0, 4, 9, 3, 5, 6]     # 9 and -1 are no pages; 3 onto itself
    for w in want:
        for s, t in ((8, 0), (1, 4), (2, 6)):
            w[t] = w[s].clone()
    gb.gformer_pages_copy(kp, vp, *(torch.tensor(x, dtype=torch.int32).cuda() for x in (src, dst)))
    torch.cuda.synchronize()
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])


@gpu
def test_pages_past_32_bit_offsets():
    page, Hkv, d, pages = 64, 8, 128, (1 << 31) // (64 * 8 * 128) + 40
    kp, vp = (torch.empty(pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gen = torch.Generator().manual_seed(6)
    k, v = (torch.randn(150, Hkv, d, generator=gen).bfloat16().cuda() for _ in range(2))
    q = torch.randn(1, 32, d, generator=gen).bfloat16().cuda()
    table = torch.tensor([[pages - 1, pages - 3, pages - 2]], dtype=torch.int32).cuda()
    zero = torch.zeros(1, dtype=torch.int32).cuda()
    gb.gformer_paged_fill(k[:149], v[:149], kp, vp, table, zero, torch.tensor([0, 149], dtype=torch.int32).cuda())
    out = torch.empty_like(q)
    gb.gformer_paged_decode(q, k[149:], v[149:], out, kp, vp, table, zero + 149, softmax_scale=0.1)
    x = dict(q=q, k=k[149:], v=v[149:], lens=[149])
    want = expect(x, [k[:149].cpu()], [v[:149].cpu()], 0.1, "bf16")
    ref.check(out, *want, "out")
    gb.gformer_pages_copy(kp, vp, table[0, :2].contiguous(), torch.tensor([pages - 4, 0], dtype=torch.int32).cuda())
    moved = torch.tensor([[pages - 4, 0, pages - 2]], dtype=torch.int32).cuda()
    again = torch.empty_like(q)
    gb.gformer_paged_decode(q, None, None, again, kp, vp, moved, zero + 150, softmax_scale=0.1)
    torch.cuda.synchronize()
    ref.check(again, *want, "out from the copies")


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_then_tokens_then_a_fork(dtype):
    """Two layers' worth of a serving run: prompts, tokens, a fork that goes its own way, a sequence freed, compaction, more
    tokens; every row against the formulas over the sequence's own keys."""
    H, Hkv, d, layers, scale = 6, 2, 64, 2, 0.125
    gen = torch.Generator().manual_seed(7)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(ref.TYPES[dtype]).cuda()
    c = PagedCache(40, 16, Hkv, d, 4, 8, layers=layers, dtype=ref.TYPES[dtype])
    for pages in (c.kpages, c.vpages):
        pages.fill_(NAN)
    c.free(c.open(33))                                   # pages 0 .. 2 come first again
    lens = [37, 50, 16]
    seqs = [c.open(n) for n in lens]
    cu = torch.tensor(ref.offsets(lens), dtype=torch.int32).cuda()
    rows = [{} for _ in range(layers)]                   # per layer: sequence -> (keys, values)
    start = torch.zeros(3, dtype=torch.int32).cuda()
    for i in range(layers):
        q, k, v = rnd(103, H, d), rnd(103, Hkv, d), rnd(103, Hkv, d)
        out = gb.gformer_packed_attn_fwd(q, k, v, torch.empty_like(q), cu, softmax_scale=scale)
        gb.gformer_paged_fill(k, v, *c.layer(i), c.table[:3], start, cu)
        ref.check(out, *ref.packed(q, k, v, None, lens, lens, scale, dtype)["out"], "prompt")
        for s, a, n in zip(seqs, ref.offsets(lens), lens):
            rows[i][s] = (k[a:a + n].cpu(), v[a:a + n].cpu())

    def tokens(live):
        c.reserve(live)
        for i in range(layers):
            q, k, v = rnd(4, H, d), rnd(4, Hkv, d), rnd(4, Hkv, d)
            got = gb.gformer_paged_decode(q, k, v, torch.empty_like(q), *c.layer(i), c.table, c.lens, softmax_scale=scale)
            held = [rows[i].get(s, (torch.zeros(0, Hkv, d), torch.zeros(0, Hkv, d))) for s in range(4)]
            x = dict(q=q, k=k, v=v, lens=c.lens.cpu())
            ref.check(got, *expect(x, [h[0] for h in held], [h[1] for h in held], scale, dtype), "token")
            for s in live:
                rows[i][s] = tuple(torch.cat([old, new[s:s + 1].cpu()]) for old, new in zip(rows[i][s], (k, v)))
        c.advance(live)

    for _ in range(3):
        tokens(seqs)
    fork = c.fork(seqs[1])
    for r in rows:
        r[fork] = r[seqs[1]]
    for _ in range(12):
        tokens(seqs + [fork])
    c.free(seqs[0])
    for r in rows:
        del r[seqs[0]]
    assert c.compact() > 0
    for _ in range(2):
        tokens([seqs[1], seqs[2], fork])


@gpu
def test_captured_step():
    x, ks, vs = make([300, 2000, 5], 8, 2, 128, 64, "bf16", 8)
    want = expect(x, ks, vs, 0.1, "bf16")
    out = torch.empty_like(x["q"])
    need = gb.gformer_paged_decode_workspace_bytes(3, 8, 2, 128, 0, table_width=x["table"].shape[1])
    spaces = [torch.empty(max(need, 1), dtype=torch.uint8, device="cuda") for _ in range(2)]
    graphs = []
    for ws in spaces:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            gb.gformer_paged_decode(**x, out=out, softmax_scale=0.1, workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            gb.gformer_paged_decode(**x, out=out, softmax_scale=0.1, workspace=ws)
    first = None
    for n in range(4):
        out.zero_()
        graphs[n % 2].replay()
        torch.cuda.synchronize()
        ref.check(out, *want, "replay")
        first = out.clone() if first is None else first
        assert torch.equal(out, first) and torch.equal(step(x, 0.1), first)


@gpu
def test_the_extension_module_makes_the_plain_calls(monkeypatch):
    x, ks, vs = make([300, 20], 8, 2, 64, 16, "bf16", 9)
    made, quick = [], gb._quick
    monkeypatch.setattr(gb, "_quick", lambda *a: made.append(quick(*a)) or made[-1])
    step(x, 0.1)
    pages = x["kpages"].clone(), x["vpages"].clone()
    cu, start = (torch.tensor(t, dtype=torch.int32).cuda() for t in ([0, 1, 2], [3, 5]))
    src, dst = (x["table"][0, i:i + 1].contiguous() for i in (1, 2))
    for pair in (pages, (x["kpages"], x["vpages"])):
        gb.gformer_paged_fill(x["k"], x["v"], *pair, x["table"], start, cu)
        gb.gformer_pages_copy(*pair, src, dst)
        monkeypatch.setattr(gb, "_quick", lambda *a: False)     # the second time in Python
    assert made == [True] * 3
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(pages, (x["kpages"], x["vpages"])))


# ---- calls whose sequences may be long, and whose rows are many --------------------------------------

class Split(ctypes.Structure):
    _fields_ = [("chunk", ctypes.c_int), ("splits", ctypes.c_int)]


def test_chunks_cover_every_length():
    """The library's own cut of a sequence, from one row to more than any launch has, and up to the longest sequence."""
    cut = getattr(gb.lib(), "_ZN7gformer11paged_splitEiiil")
    cut.restype, cut.argtypes = Split, [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int64]
    for B in (1, 2, 32, 191, 192, 193, 1535, 1536, 1537, 8192, 1 << 20, 2 ** 31 - 1):
        for H, Hkv in ((1, 1), (8, 8), (32, 8), (40, 2), (32, 32), (2 ** 31 - 1, 1), (2 ** 31 - 1, 2 ** 31 - 1)):
            for room in (0, 1, 63, 64, 129, 5000, 1 << 20, 1 << 24, (1 << 29) - 1, 1 << 30):
                s = cut(B, H, Hkv, room)
                what = (B, H, Hkv, room, s.chunk, s.splits)
                assert 128 <= s.chunk <= max(128, -(-room // 64) * 64) and s.chunk % 64 == 0, what
                assert s.splits >= 1 and s.chunk * s.splits >= room and s.chunk * (s.splits - 1) <= max(room - 1, 0), what
                assert s.splits == 1 or B * Hkv * -(-(H // Hkv) // 16) * s.splits < 2 * 1536, what


@gpu
def test_many_rows_over_a_table_of_many_pages():
    """Room for 2^28 tokens in each of 1600 rows of 8 key heads; three of them are in use."""
    B, H, Hkv, d, page, width = 1600, 8, 8, 64, 65536, 4096
    gen = torch.Generator().manual_seed(12)
    rnd = lambda *s: torch.randn(*s, generator=gen).bfloat16()
    lens = {0: 40, 801: 0, 1599: 700}
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    kp, vp = (torch.full((3, Hkv, page, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    held = torch.full((B,), -1, dtype=torch.int32)
    ks, vs = [], []
    for place, (b, n) in enumerate(lens.items()):
        table[b, 0], held[b] = 2 - place, n
        ks.append(rnd(n, Hkv, d))
        vs.append(rnd(n, Hkv, d))
        kp[2 - place, :, :n], vp[2 - place, :, :n] = ks[-1].transpose(0, 1).cuda(), vs[-1].transpose(0, 1).cuda()
    rows = list(lens)
    x = dict(q=rnd(B, H, d).cuda(), k=rnd(B, Hkv, d).cuda(), v=rnd(B, Hkv, d).cuda(), kpages=kp, vpages=vp, table=table, lens=held.cuda())
    got = step(x, 0.125)
    want = expect({**x, **{n: x[n][rows] for n in "qkv"}, "lens": held[rows]}, ks, vs, 0.125, "bf16")
    ref.check(got[rows], *want, "out")
    idle = torch.ones(B, dtype=torch.bool)
    idle[rows] = False
    assert not got[idle.cuda()].any()
    for place, (b, n) in enumerate(lens.items()):        # the new token is in its slot
        assert torch.equal(kp[2 - place, :, n], x["k"][b]) and torch.equal(vp[2 - place, :, n], x["v"][b])


def test_launches_stay_within_what_one_may_have():
    """A launch has less than 2^32 threads, of which a workgroup has 256; a decode step has one for every 16 query heads of a key head (two for
    20, so four a row with two key heads).  The largest call of each kind is refused for its null
    pointer alone."""
    most = (2 ** 32 - 1) // 256
    for B, H, Hkv, status in ((most // 32, 32, 32, 1), (most // 32 + 1, 32, 32, 2), (most // 8, 32, 8, 1), (most // 8 + 1, 32, 8, 2), (most // 4, 40, 2, 1),
                              (most // 4 + 1, 40, 2, 2), (2 ** 31 - 1, 2 ** 31 - 1, 1, 2), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 2)):
        assert decode(q=0, B=B, H=H, Hkv=Hkv) == status, (B, H, Hkv)
    p = gb.make_paged_params()
    fill = lambda n, total, heads: gb.lib().gformer_paged_fill(0, *(i * A for i in range(2, 8)), n, total, heads, 64, 9, 4, ctypes.byref(p), None)
    for n, total, heads in ((most // 32 - 1, 8, 32), (most - 1, 8, 1), (1, 1 << 28, most // ((1 << 28) // 32 + 2))):
        assert fill(n, total, heads) == gb.GF_ERR_INVALID_ARG
    for n, total, heads in ((most // 32, 8, 32), (most, 8, 1), (1, 1 << 28, most // ((1 << 28) // 32 + 2) + 1), (1 << 30, 8, 2 ** 31 - 1)):
        assert fill(n, total, heads) == gb.GF_ERR_UNSUPPORTED
    copy = lambda n, heads: gb.lib().gformer_pages_copy(0, 2 * A, 3 * A, 4 * A, n, heads, 64, 9, ctypes.byref(p), None)
    assert copy(most // 256, 256) == copy(most, 1) == gb.GF_ERR_INVALID_ARG
    assert copy(most // 256 + 1, 256) == copy(most + 1, 1) == copy(2 ** 31 - 1, 2 ** 31 - 1) == gb.GF_ERR_UNSUPPORTED


def test_dense_rows_are_as_long_as_strided_ones_may_be():
    p = gb.make_paged_params()
    for d in (64, 128):
        heads = (1 << 20) // d
        for h, status in ((heads, gb.GF_ERR_INVALID_ARG), (heads + 1, gb.GF_ERR_UNSUPPORTED)):
            assert decode(q=0, H=h, Hkv=1, d=d) == decode(q=0, H=h, Hkv=h, d=d) == status
            assert gb.lib().gformer_paged_fill(0, *(i * A for i in range(2, 8)), 2, 5, h, d, 9, 4, ctypes.byref(p), None) == status


def test_a_fork_whose_copy_fails_changes_nothing(monkeypatch):
    def fail(*_):
        raise gb.GformerError(4, "no device")
    c = cache()
    a = c.open(13)
    before = (list(c._held), list(c._free), [list(p or []) for p in c._pages], list(c._len))
    monkeypatch.setattr(gb, "gformer_pages_copy", fail)
    with pytest.raises(gb.GformerError):
        c.fork(a)
    assert before == (c._held, c._free, [list(p or []) for p in c._pages], c._len)
    Copies(monkeypatch)
    assert c.pages(c.fork(a)) == [0, 2]


# ---- what the books send to the device ---------------------------------------------------------------

def rows(c):
    return [(p or []) + [-1] * (c.max_pages - len(p or [])) for p in c._pages]


def test_table_and_lengths_follow_the_books(monkeypatch):
    Copies(monkeypatch)
    rng, c, live = random.Random(11), cache(n_pages=24, max_seqs=7), []
    for _ in range(600):
        try:
            what = rng.choice(["open", "fork", "free", "reserve", "step", "step", "compact"])
            if what == "open":
                live.append(c.open(rng.randint(0, 40)))
            elif what == "fork" and live:
                live.append(c.fork(rng.choice(live)))
            elif what == "free" and live:
                c.free(live.pop(rng.randrange(len(live))))
            elif what in ("reserve", "step") and live:
                some = rng.sample(live, rng.randint(1, len(live)))
                c.reserve(some)
                if what == "step":
                    c.advance(some)
            elif what == "compact":
                c.compact()
        except (RuntimeError, ValueError):
            pass
        assert c.table.tolist() == rows(c) and c.lens.tolist() == c._len


def test_a_change_sends_what_changed(monkeypatch):
    """The rows of other sequences, marked here, are not written again."""
    Copies(monkeypatch)
    c = cache()
    a, b = c.open(15), c.open(9)
    mark = 77
    c.table[a] = mark
    c.reserve([b])
    c.advance([b])
    c.free(c.fork(b))
    for _ in range(7):
        c.reserve([b])                                   # the last one takes a page
        c.advance([b])
    assert c.table[a].tolist() == [mark] * 5 and c.table[b].tolist() == c.pages(b) + [-1] * 2 and c.length(b) == 17
    sent = []
    monkeypatch.setattr(c, "_send", lambda numbers, dtype, send=c._send: sent.append(len(numbers)) or send(numbers, dtype))
    c.advance([a])
    c.reserve([b])
    assert sent == []                                    # lengths alone
    c.reserve([a])
    assert sent == [1, 1] and c.table[a].tolist() == [mark, mark, c.pages(a)[2], mark, mark]


def test_a_change_that_the_device_has_no_memory_for_is_none(monkeypatch):
    Copies(monkeypatch)
    c = cache()
    a, b = c.open(16), c.open(3)
    before = (list(c._held), list(c._free), [list(p or []) for p in c._pages], list(c._len), c.table.tolist(), c.lens.tolist())

    def fail(*_):
        raise torch.OutOfMemoryError("none left")
    monkeypatch.setattr(c, "_send", fail)
    for call in (lambda: c.open(9), lambda: c.fork(a), lambda: c.fork(b), lambda: c.reserve([a, b]), lambda: c.free(a)):
        with pytest.raises(torch.OutOfMemoryError):
            call()
        assert before == (c._held, c._free, [list(p or []) for p in c._pages], c._len, c.table.tolist(), c.lens.tolist())


@gpu
def test_a_step_waits_for_nothing():
    """Bookkeeping behind 50 large products returns while they run, and takes its place behind them."""
    c = PagedCache(300, 8, 2, 64, 40, 512)
    seqs = [c.open(7) for _ in range(32)]
    x = torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    y = torch.empty_like(x)
    torch.mm(x, x, out=y)
    c.advance(seqs)
    c.free(seqs.pop())
    torch.cuda.synchronize()
    done = torch.cuda.Event()
    for _ in range(50):
        torch.mm(x, x, out=y)
    done.record()
    was = c.table.clone(), c.lens.clone()                # read behind the products, in front of the changes
    c.reserve(seqs)
    c.advance(seqs)
    new = c.open(20)
    c.fork(new)
    c.free(seqs.pop(0))
    assert not done.query()
    torch.cuda.synchronize()
    assert was[0][1].tolist() == [1] + [-1] * 511 and was[1].tolist() == [8] * 31 + [-1] * 9
    assert c.table.tolist() == rows(c) and c.lens.tolist() == c._len and c._len[new] == 20


def test_scales_that_overflow_are_refused():
    assert all(decode(p=wrong(softmax_scale=x), width=64, ws=0) == 1 for x in (3e38, -3e38, NAN, float("inf")))
    assert all(decode(p=wrong(softmax_scale=x), width=64, ws=0) == 3 for x in (2.0 ** 127, -2.0 ** 127, 0.0, 1e-40))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_scales_of_large_scores(dtype):
    x, _, _ = make([40, 300], 4, 2, 64, 16, dtype, 3, fill=0.0)
    y = {n: t.clone() for n, t in x.items()}             # each step writes its token into pages of its own
    want, by = step(x, 0.125), 2.0 ** 57
    for n in ("q", "k", "kpages"):
        y[n] = y[n] * by
    assert torch.equal(step(y, 0.125 / by / by), want)


def test_numbers_past_32_bits_are_refused():
    """... not cut to what is left of them: a bound of 2^32 + 5 tokens, say, to one of 5."""
    b = gb.gformer_paged_decode_workspace_bytes
    for kw in (dict(max_len=2 ** 32 + 5, table_width=4), dict(max_len=-2 ** 32, table_width=4), dict(max_len=5, table_width=2 ** 32 + 4)):
        with pytest.raises(ValueError, match="32 bits"):
            b(1, 4, 2, 64, **kw)
    with pytest.raises(ValueError, match="n_seqs"):
        gb.gformer_packed_attn_bwd_workspace_bytes(8, 8, 2 ** 32 + 1, 2, 2, 64)
    meta = lambda *shape, dtype=torch.int32: torch.empty(*shape, dtype=dtype, device="meta")
    with pytest.raises(ValueError, match="table"):
        gb._numbers(meta(1), (1, None), table=meta(1, 2 ** 32 + 4))
    with pytest.raises(ValueError, match="kpages"):
        gb._tensors(meta(1, dtype=torch.bfloat16), 4, kpages=meta(2 ** 31, 1, 8, 64, dtype=torch.bfloat16))


@gpu
def test_a_bound_past_32_bits_is_refused():
    x, _, _ = make([40], 4, 2, 64, 16, "bf16", 3)
    for bound in (2 ** 32, 2 ** 32 + 5):
        with pytest.raises(ValueError, match="max_len"):
            step(x, 0.125, max_len=bound)


@gpu
def test_the_books_do_not_change_while_a_graph_is_captured():
    """A replay would send memory that has long been another's; the calls say so, and the capture goes on."""
    c = PagedCache(20, 8, 2, 64, 4, 8)
    a, b = c.open(8), c.open(3)
    before = (list(c._held), list(c._free), [list(p or []) for p in c._pages], list(c._len), c.table.tolist(), c.lens.tolist())
    x = torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1)
        for call in (lambda: c.advance([b]), lambda: c.reserve([a]), lambda: c.open(0), lambda: c.open(9), lambda: c.fork(a), lambda: c.fork(b),
                     lambda: c.free(a)):
            with pytest.raises(RuntimeError, match="captured"):
                call()
        x.add_(1)
    for n in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        assert (x == 2 * n).all()
    assert before == (c._held, c._free, [list(p or []) for p in c._pages], c._len, c.table.tolist(), c.lens.tolist())
    c.advance([b])
    assert c.lens.tolist() == [8, 4, -1, -1]


@gpu
def test_the_largest_launch():
    """As many rows of 32 heads as a launch holds, three of them in use."""
    H, d, page, B = 32, 64, 8, (2 ** 32 - 1) // 256 // 32
    gen = torch.Generator("cuda").manual_seed(82)
    q, k, v = (torch.randn(B, H, d, device="cuda", generator=gen, dtype=torch.bfloat16) for _ in range(3))
    kp, vp = (torch.randn(3, H, page, d, device="cuda", generator=gen, dtype=torch.bfloat16) for _ in range(2))
    rows, lens = [0, 300000, B - 1], [0, 7, 4]
    table = torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    held = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    for i, (b, n) in enumerate(zip(rows, lens)):
        table[b, 0], held[b] = i, n
    ks, vs = ([x[i, :, :n].transpose(0, 1).cpu() for i, n in enumerate(lens)] for x in (kp, vp))
    out = torch.full_like(q, 7.0)
    gb.gformer_paged_decode(q, k, v, out, kp, vp, table, held, softmax_scale=0.125)
    torch.cuda.synchronize()
    ref.check(out[rows], *expect(dict(q=q[rows], k=k[rows], v=v[rows], lens=held[rows].cpu()), ks, vs, 0.125, "bf16"), "out")
    out[rows] = 0
    assert not out.any()
    for i, (b, n) in enumerate(zip(rows, lens)):
        assert torch.equal(kp[i, :, n], k[b]) and torch.equal(vp[i, :, n], v[b])
