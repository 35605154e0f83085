"""A paged cache of 4 bits a value and rotary positions, as a program calls them, beside the same operators in elementary
torch operations.

    own                 False: run() computes the plain form; True: it calls the library
    listed()            the fixed cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program holds before the call (device tensors, page table)
    run(state)          one pass; returns its outputs
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   the same outputs in 64 bits

Five kinds of call:
    prompt  new tokens' keys and values into the cache, and every key and value of their sequences out of it, as a prompt that
            goes on behind cached tokens needs them
    read    cached tokens out of the cache alone
    decode  one new token of every sequence over the cache, and what the cache then holds of it
    rotary  queries and keys turned by their positions
    train   the same with its gradients, through the differentiable wrapper

A row of the cache, one token of one head, is d / 2 bytes of codes (channel c in bits 4 (c % 2) .. of byte c / 2), and behind
them for each 32 channels a scale and a lowest value in bf16: code n stands for low + scale n.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
GROUP = 32


def _text(v):
    return ",".join(str(int(x)) for x in v)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _named(name, case):
    return case if name is None else {"name": name, **case}


def _cached(kind, dtype, Hkv, d, lens, held, page, tail=0, name=None):
    """lens: rows of each sequence in the call; held: tokens of each that are in the cache before it (prompt) or that the rows
    come behind (read); tail: rows behind the last sequence, as a batch padded to a fixed size has them."""
    return _named(name, {"kind": kind, "dtype": dtype, "Hkv": Hkv, "d": d, "lens": _text(lens), "held": _text(held), "page": page,
                         "tail": tail})


def _decode(dtype, H, Hkv, d, lens, page, name=None):
    """lens: tokens of each sequence that are in the cache already."""
    return _named(name, {"kind": "decode", "dtype": dtype, "H": H, "Hkv": Hkv, "d": d, "lens": _text(lens), "page": page})


def _rotary(kind, dtype, H, Hkv, d, rot, interleaved, lens, held, stretch=1.0, by_row=False, tail=0, name=None):
    """rot: channels of a head that turn; lens, held: rows of each sequence and the position of its first; stretch: how many times
    longer than the trained length the positions may get; by_row: the rows' positions in a tensor, not from offsets."""
    return _named(name, {"kind": kind, "dtype": dtype, "H": H, "Hkv": Hkv, "d": d, "rot": rot, "interleaved": interleaved,
                         "lens": _text(lens), "held": _text(held), "stretch": stretch, "by_row": by_row, "tail": tail})


def listed():
    return [
        # One short prompt of a 12-head layer into the cache and back: the smallest call, all latency.
        _cached("prompt", "bf16", 12, 64, [128], [0], 16, name="prompt_one"),
        # A serving engine's step: whole prompts, chunks that go on behind cached tokens, a single token, a sequence with nothing new.
        _cached("prompt", "bf16", 8, 128, [1531, 512, 77, 1, 2048, 300, 0, 640, 129, 1024, 33, 911],
                [0, 1536, 0, 1699, 0, 913, 50, 0, 1172, 0, 5, 1136], 64, tail=200, name="prompts_ragged"),
        # Long shared prefixes come out of the cache for the prompts behind them: the largest read.
        _cached("read", "bf16", 8, 128, [32767, 20000, 4099], [0, 0, 1021], 128, name="read_long"),
        # Full precision, every head with keys of its own, small pages.
        _cached("read", "f32", 16, 64, [2048, 1000, 17, 3000, 1], [0, 24, 0, 77, 4095], 32, tail=31, name="read_f32"),
        # One token for one user of a 12-head model: latency.
        _decode("bf16", 12, 12, 64, [2047], 16, name="decode_one"),
        # One token for a batch of users whose contexts differ, grouped heads.
        _decode("bf16", 32, 8, 128,
                [8191, 4096, 77, 1300, 2500, 6000, 1, 0, 3333, 511, 512, 7100, 900, 4800, 64, 2222,
                 5000, 127, 128, 6789, 1024, 3100, 40, 8000, 1999, 700, 4321, 260, 7777, 15, 5555, 1600],
                64, name="decode_batch"),
        # Many users with long contexts, which is what a small cache is for: the largest pass over it.
        _decode("bf16", 32, 8, 128, [32767, 32768, 20000, 31111, 16384, 30001, 25000, 32000], 128, name="decode_long"),
        # Full precision, every head with keys of its own.
        _decode("f32", 16, 16, 64, [2048, 1000, 3000, 17, 4095, 1], 32, name="decode_f32"),
        # The new tokens of a few users: the smallest turn, all latency.
        _rotary("rotary", "bf16", 12, 12, 64, 64, True, [1] * 4, [2047, 16, 0, 900], by_row=True, name="rotary_tokens"),
        # Packed prompts of the 32-head model with shared key heads, some behind cached tokens.
        _rotary("rotary", "bf16", 32, 8, 128, 128, False, [1531, 512, 77, 1, 2048, 300, 0, 640, 129, 1024, 33, 911],
                [0, 1536, 0, 1699, 0, 913, 50, 0, 1172, 0, 5, 1136], tail=200, name="rotary_prompts"),
        # Half of every head turns, far positions of a stretched context, full precision.
        _rotary("rotary", "f32", 16, 4, 128, 64, True, [3001, 1000], [1000003, 77], stretch=8.0, name="rotary_far"),
        # A training step's turn over packed documents and its way back.
        _rotary("train", "bf16", 32, 8, 128, 128, False, [4096, 3001, 1095], [0, 0, 0], tail=64, name="rotary_train"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# what a drawn case may cost
_LARGEST = {"prompt": "prompts_ragged", "read": "read_long", "decode": "decode_long", "rotary": "rotary_prompts", "train": "rotary_train"}
_MOST_PADDED = 8 * 8 * 32769 * 128     # values of keys that the plain form of a decode step may hold, with its padding


def _shared(rng, H):
    return rng.choice([x for x in (1, 2, 4, 8, H) if H % x == 0])


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "read", "decode", "decode", "decode", "rotary", "rotary", "train"])
    d = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    top = next(work(c) for c in listed() if c["name"] == _LARGEST[kind])
    fits = lambda case: all(work(case)[x] <= top[x] for x in top)
    H = rng.choice([8, 12, 16, 32])
    if kind == "decode":
        Hkv = _shared(rng, H)
        B, longest = _log_int(rng, 1, 48), _log_int(rng, 16, 32768)
        while True:
            case = _decode(dtype, H, Hkv, d, [rng.choice([longest, rng.randint(0, longest)]) for _ in range(B)],
                           rng.choice([16, 32, 64, 128, 256]))
            if fits(case) and B * Hkv * (longest + 256) * d <= _MOST_PADDED:
                return case
            B, longest = max(1, B // 2), max(1, longest * 2 // 3)
    n, longest = _log_int(rng, 1, 16), _log_int(rng, 16, 32768 if kind == "read" else 8192)
    tail = rng.choice([0, 0, rng.randint(1, 200)])
    far = rng.choice([longest, longest, 1 << 20]) if kind in ("rotary", "train") else longest
    rot = rng.choice([d, d, d // 2, d // 4])
    interleaved, stretch, by_row = rng.random() < 0.5, rng.choice([1.0, 1.0, 4.0, 8.0]), rng.random() < 0.5
    Hkv = _shared(rng, H) if kind in ("rotary", "train") else rng.choice([1, 2, 4, 8, 12, 16])
    while True:
        lens = [longest] + [rng.choice([1, rng.randint(0, longest)]) for _ in range(n - 1)]
        held = [rng.randint(0, far) * rng.randint(0, 1) for _ in lens]
        if kind in ("rotary", "train"):
            case = _rotary(kind, dtype, H, Hkv, d, rot, interleaved, lens, held, stretch, by_row, 0 if by_row else tail)
        else:
            case = _cached(kind, dtype, Hkv, d, lens, held, rng.choice([8, 16, 32, 64, 128, 256]), tail)
        if fits(case):
            return case
        n, longest = (n // 2, longest) if n > 1 else (n, longest * 2 // 3)
        far = min(far, max(longest, 1)) if kind in ("prompt", "read") else far


# ---- a cache of 4 bits in elementary operations ------------------------------------------------
def _down(x, up):
    """The nearest bf16 value at or below (up: above) finite values in 64 bits."""
    y = x.to(torch.float32).to(torch.bfloat16)
    bits = y.view(torch.int16)
    far = (y.double() < x) if up else (y.double() > x)
    away = (y > 0) if up else (y < 0)      # whether the next value's magnitude is larger
    # from zero the next one is the smallest of its sign
    least = torch.full_like(bits, 1) if up else torch.full_like(bits, -32767)
    moved = torch.where(y == 0, least, torch.where(away, bits + 1, bits - 1))
    return torch.where(far, moved, bits).view(torch.bfloat16)


def _quantised(x):
    """[..., d] -> rows of the cache [..., d / 2 + d / 8] in bytes."""
    d = x.shape[-1]
    x = x.double().unflatten(-1, (d // GROUP, GROUP))
    sound = (x.abs() < 2.0 ** 127).all(-1)
    x = torch.where(sound[..., None], x, 0.0)
    low = _down(x.amin(-1), up=False)
    scale = _down((x.amax(-1) - low.double()) / 15.0, up=True)
    step = scale.double()[..., None]
    codes = torch.where(step > 0, torch.round((x - low.double()[..., None]) / torch.where(step > 0, step, 1.0)), 0.0)
    codes = codes.to(torch.uint8).flatten(-2)
    nan = torch.full_like(low, math.nan)
    pairs = torch.stack([torch.where(sound, scale, nan), torch.where(sound, low, nan)], -1).flatten(-2)
    return torch.cat([codes[..., ::2] | codes[..., 1::2] << 4, pairs.view(torch.uint8)], -1)


def _values(rows):
    """Rows of the cache -> what they stand for, in 32 bits."""
    d = rows.shape[-1] * 8 // 5
    codes = torch.stack([rows[..., :d // 2] & 15, rows[..., :d // 2] >> 4], -1).flatten(-2).float().unflatten(-1, (d // GROUP, GROUP))
    pairs = rows[..., d // 2:].contiguous().view(torch.bfloat16).float().unflatten(-1, (d // GROUP, 2))
    return (pairs[..., 1:] + pairs[..., :1] * codes).flatten(-2)


# ---- inputs --------------------------------------------------------------------------------
def _offsets(lens):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device="cuda")


def _table(gen, lens, page, spare):
    """A page table for sequences of up to `lens` tokens: every page anywhere in the cache, each used once."""
    need = [-(-x // page) for x in lens]
    pages = sum(need) + spare
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((len(lens), max(max(need), 1)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def _frequencies(rot, stretch):
    """Angles per position of each pair of channels: base^(-2 i / rot), and for a stretched context slow pairs, which do not turn
    once in the 4096 positions of the trained length, slowed by `stretch`, fast ones kept, those between by a ramp."""
    i = torch.arange(0, rot, 2, dtype=torch.float64)
    f = 10000.0 ** (-i / rot)
    turns = 4096 * f / (2 * math.pi)
    keep = ((turns - 1) / 31).clamp(0, 1)
    return (f * keep + f / stretch * (1 - keep)).float().to("cuda")


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dt, d, kind = DTYPES[case["dtype"]], case["d"], case["kind"]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(dt)

    def pages(n, heads, page):
        """A cache filled with what quantising keys or values leaves."""
        out = torch.empty(n, heads, page, d * 5 // 8, dtype=torch.uint8, device="cuda")
        for part in out.split(max(1, (1 << 24) // (heads * page * d))):
            part.copy_(_quantised(normal(*part.shape[:3], d)))
        return out

    s = dict(case)
    lens = _ints(case["lens"])
    s["n"], s["longest"] = len(lens), max(lens)
    if kind == "decode":
        s["scale"] = 1.0 / math.sqrt(d)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["table"], n = _table(gen, [x + 1 for x in lens], case["page"], 3)
        s["kpages"], s["vpages"] = (pages(n, case["Hkv"], case["page"]) for _ in range(2))
        s["q"], s["k"], s["v"] = normal(len(lens), case["H"], d), normal(len(lens), case["Hkv"], d), normal(len(lens), case["Hkv"], d)
        s["out"], s["kheld"], s["vheld"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
        s["cu"] = torch.arange(len(lens) + 1, dtype=torch.int32, device="cuda")     # one row each
        return s
    held, rows = _ints(case["held"]), sum(lens) + case["tail"]
    s["cu"], s["start"] = _offsets(lens), torch.tensor(held, dtype=torch.int32, device="cuda")
    if kind in ("prompt", "read"):
        s["table"], n = _table(gen, [a + b for a, b in zip(lens, held)], case["page"], 3)
        s["kpages"], s["vpages"] = (pages(n, case["Hkv"], case["page"]) for _ in range(2))
        if kind == "prompt":
            # the keys' and values' part of one fused projection's output, as a layer has it
            kv = normal(rows, 2 * case["Hkv"], d)
            s["k"], s["v"] = kv[:, :case["Hkv"]], kv[:, case["Hkv"]:]
            s["from"], s["cu_all"] = torch.zeros_like(s["start"]), _offsets([a + b for a, b in zip(lens, held)])
            rows = sum(lens) + sum(held) + case["tail"]
        s["kout"], s["vout"] = (torch.zeros(rows, case["Hkv"], d, dtype=dt, device="cuda") for _ in range(2))
        return s
    s["freqs"] = _frequencies(case["rot"], case["stretch"])
    s["factor"] = 1.0 if case["stretch"] == 1.0 else 0.1 * math.log(case["stretch"]) + 1.0
    if case["by_row"]:
        s["positions"] = torch.cat([torch.arange(a, a + n, dtype=torch.int32) for a, n in zip(held, lens)]).to("cuda")
    qkv = normal(rows, case["H"] + 2 * case["Hkv"], d)
    s["q"], s["k"] = qkv[:, :case["H"]], qkv[:, case["H"]:case["H"] + case["Hkv"]]
    if kind == "train":
        s["q"], s["k"] = (x.contiguous().requires_grad_(True) for x in (s["q"], s["k"]))
        s["dq"], s["dk"] = normal(rows, case["H"], d), normal(rows, case["Hkv"], d)
    else:
        s["qout"], s["kout"] = (torch.zeros(x.shape, dtype=dt, device="cuda") for x in (s["q"], s["k"]))
    return s


# ---- the plain forms -----------------------------------------------------------------------
def _places(cu, rows):
    """(sequence, position, in one) of every row of a packed tensor."""
    row = torch.arange(rows, device=cu.device)
    seq = torch.searchsorted(cu[1:].long(), row, right=True)
    inside = seq < cu.numel() - 1
    seq = seq.clamp(max=cu.numel() - 2)
    return seq, torch.where(inside, row - cu.long()[seq], 0), inside


def _slots(s, cu, start, rows):
    seq, pos, inside = _places(cu, rows)
    seq, pos = seq[inside], pos[inside] + start.long()[seq[inside]]
    return inside, s["table"][seq, pos // s["page"]].long(), pos % s["page"]


def _plain_fill(s, x, pages):
    inside, page, slot = _slots(s, s["cu"], s["start"], x.shape[0])
    pages[page, :, slot] = _quantised(x[inside])


def _plain_read(s, pages, cu, start, out):
    inside, page, slot = _slots(s, cu, start, out.shape[0])
    out[inside] = _values(pages[page, :, slot]).to(out.dtype)


def _plain_decode(s):
    B, H, Hkv, d, page = s["n"], s["H"], s["Hkv"], s["d"], s["page"]
    t, users = s["lens"].long(), torch.arange(s["n"], device="cuda")
    at = s["table"][users, t // page].long()
    for x, pages in ((s["k"], s["kpages"]), (s["v"], s["vpages"])):
        pages[at, :, t % page] = _quantised(x)
    held = [_values(pages[at, :, t % page]).to(s["q"].dtype) for pages in (s["kpages"], s["vpages"])]
    width = s["table"].shape[1]
    rows = s["table"].clamp(min=0).long()
    k, v = (_values(pages[rows].transpose(1, 2).reshape(B, Hkv, width * page, -1)) for pages in (s["kpages"], s["vpages"]))
    q = s["q"].float().view(B, Hkv, H // Hkv, d)
    hidden = torch.arange(width * page, device="cuda")[None] > t[:, None]
    scores = ((q @ k.transpose(-1, -2)) * s["scale"]).masked_fill(hidden[:, None, None], -math.inf)
    p = (scores - scores.amax(-1, keepdim=True)).exp()
    out = (p / p.sum(-1, keepdim=True)) @ v.masked_fill(hidden[:, None, :, None], 0.0)
    return out.view(B, H, d).to(s["q"].dtype), *held


def _plain_turn(s, x, pos):
    rot, half = s["rot"], s["rot"] // 2
    angle = pos.double()[:, None] * s["freqs"].double()
    cos, sin = ((f(angle) * s["factor"]).float()[:, None] for f in (torch.cos, torch.sin))
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if s["interleaved"] else (x[..., :half], x[..., half:rot])
    a, b = a.float(), b.float()
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.stack(y, -1).flatten(-2) if s["interleaved"] else torch.cat(y, -1)
    return torch.cat([y, x[..., rot:].float()], -1).to(x.dtype)


def _plain_rotary(s):
    if s["by_row"]:
        return [_plain_turn(s, x, s["positions"]) for x in (s["q"], s["k"])]
    seq, pos, inside = _places(s["cu"], s["q"].shape[0])
    pos = pos + s["start"].long()[seq]
    return [torch.where(inside[:, None, None], _plain_turn(s, x, pos), torch.zeros((), dtype=x.dtype, device="cuda")) for x in (s["q"], s["k"])]


def run(s):
    kind = s["kind"]
    if own:
        from paper_2412_19829_amd import binding as gb
    if kind in ("prompt", "read"):
        if kind == "prompt":
            if own:
                gb.gformer_paged_fill_q4(s["k"], s["v"], s["kpages"], s["vpages"], s["table"], s["start"], s["cu"])
            else:
                _plain_fill(s, s["k"], s["kpages"])
                _plain_fill(s, s["v"], s["vpages"])
        cu, start = (s["cu_all"], s["from"]) if kind == "prompt" else (s["cu"], s["start"])
        if own:
            gb.gformer_paged_read_q4(s["kpages"], s["vpages"], s["kout"], s["vout"], s["table"], start, cu)
        else:
            _plain_read(s, s["kpages"], cu, start, s["kout"])
            _plain_read(s, s["vpages"], cu, start, s["vout"])
        return s["kout"], s["vout"]
    if kind == "decode":
        if not own:
            return _plain_decode(s)
        gb.gformer_paged_decode_q4(s["q"], s["k"], s["v"], s["out"], s["kpages"], s["vpages"], s["table"], s["lens"],
                                   max_len=s["longest"] + 1, softmax_scale=s["scale"])
        gb.gformer_paged_read_q4(s["kpages"], s["vpages"], s["kheld"], s["vheld"], s["table"], s["lens"], s["cu"])
        return s["out"], s["kheld"], s["vheld"]
    where = {"positions": s["positions"]} if s["by_row"] else {"cu": s["cu"], "start": s["start"]}
    if kind == "rotary":
        if not own:
            return tuple(_plain_rotary(s))
        gb.gformer_rotary(s["q"], s["k"], s["qout"], s["kout"], s["freqs"], interleaved=int(s["interleaved"]), factor=s["factor"], **where)
        return s["qout"], s["kout"]
    if own:
        from paper_2412_19829_amd.autograd import gformer_rotary_positions
        q, k = gformer_rotary_positions(s["q"], s["k"], s["freqs"], interleaved=int(s["interleaved"]), factor=s["factor"], **where)
    else:
        q, k = _plain_rotary(s)
    return (q.detach(), k.detach(), *torch.autograd.grad((q, k), (s["q"], s["k"]), (s["dq"], s["dk"])))


# ---- what a pass cannot do without ----------------------------------------------------------
def work(case):
    size, d, lens = BYTES[case["dtype"]], case["d"], _ints(case["lens"])
    row = d * 5 // 8
    n = sum(lens)
    if case["kind"] == "decode":
        H, Hkv, seen = case["H"], case["Hkv"], n + len(lens)
        # cached rows, the new token's in, into its slot, out of it and out again, queries in and results out, the pages' numbers
        moved = 2 * n * Hkv * row + 2 * len(lens) * Hkv * (2 * d * size + row) + 2 * len(lens) * H * d * size
        return {"bytes": moved + 4 * sum(-(-(x + 1) // case["page"]) + 1 for x in lens), "flops": 4 * seen * H * d}
    if case["kind"] in ("prompt", "read"):
        held = sum(_ints(case["held"])) if case["kind"] == "prompt" else 0
        read = 2 * (n + held) * case["Hkv"] * (row + d * size)
        fill = 2 * n * case["Hkv"] * (row + d * size) if case["kind"] == "prompt" else 0
        # a value read is a product and a sum; one written two comparisons, a difference, a quotient and a rounding
        return {"bytes": read + fill, "flops": 2 * (2 * (n + held) + (5 * n if fill else 0)) * case["Hkv"] * d}
    heads = case["H"] + case["Hkv"]
    passes = 2 if case["kind"] == "train" else 1
    return {"bytes": passes * 2 * n * heads * d * size, "flops": passes * 3 * n * heads * case["rot"]}


# ---- the same in 64 bits --------------------------------------------------------------------
def _exact_held(row, d):
    """What rows of bytes stand for."""
    out = torch.empty(*row.shape[:-1], d, dtype=torch.float64, device=row.device)
    pairs = row[..., d // 2:].contiguous().view(torch.bfloat16).double()
    for g in range(d // 32):
        code = row[..., 16 * g:16 * g + 16].double()
        high = torch.floor(code / 16)
        scale, low = pairs[..., 2 * g, None], pairs[..., 2 * g + 1, None]
        out[..., 32 * g:32 * g + 32:2] = low + scale * (code - 16 * high)
        out[..., 32 * g + 1:32 * g + 32:2] = low + scale * high
    return out


def _exact_stored(x):
    """What [..., d] values stand for once they have been stored: the lowest bf16 at or below each 32 channels' smallest, the smallest
    bf16 step whose 15 reach their largest, and the nearest of the 16 values (of two as near, the one of even code)."""
    d = x.shape[-1]
    x = x.double()
    out = torch.empty_like(x)
    for g in range(d // 32):
        part = x[..., 32 * g:32 * g + 32]
        least, most = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values
        low = _exact_grid(least, torch.floor)
        step = _exact_grid((most - low) / 15, torch.ceil)
        at = (part - low) / torch.where(step > 0, step, 1.0)
        n = torch.floor(at)
        n = n + ((at - n > 0.5) | ((at - n == 0.5) & (n % 2 == 1)))
        out[..., 32 * g:32 * g + 32] = low + step * torch.where(step > 0, n, 0.0)
    return out


def _exact_grid(x, to):
    """x moved by `to` onto the values of 8 significant bits."""
    _, e = torch.frexp(x)
    unit = torch.exp2((e.double() - 8).clamp(min=-133))
    return to(x / unit) * unit


def exact(case, seed):
    s = prepare(case, seed)
    kind, d, lens = case["kind"], case["d"], _ints(case["lens"])
    if kind in ("prompt", "read"):
        held, page = _ints(case["held"]), case["page"]
        outs = []
        for pages, new, out in ((s["kpages"], s.get("k"), s["kout"]), (s["vpages"], s.get("v"), s["vout"])):
            full = torch.zeros(out.shape, dtype=torch.float64, device="cuda")
            stored = _exact_stored(new) if new is not None else None
            a = c = 0
            for b, (n, h) in enumerate(zip(lens, held)):
                first, last = (0, h) if new is not None else (h, h + n)       # tokens that come out of the cache as it was
                for p in range(first // page, -(-last // page) if last > first else 0):
                    lo, hi = max(first, p * page), min(last, (p + 1) * page)
                    if lo < hi:
                        rows = pages[int(s["table"][b, p]), :, lo - p * page:hi - p * page]
                        full[c + lo - first:c + hi - first] = _exact_held(rows, d).transpose(0, 1)
                c += last - first
                if new is not None:
                    full[c:c + n] = stored[a:a + n]
                    a, c = a + n, c + n
            outs.append(full)
        return tuple(outs)
    if kind == "decode":
        H, Hkv, page = case["H"], case["Hkv"], case["page"]
        knew, vnew = _exact_stored(s["k"]), _exact_stored(s["v"])
        out = torch.zeros(len(lens), H, d, dtype=torch.float64, device="cuda")
        for b, t in enumerate(lens):
            ids = s["table"][b, :-(-t // page)].long()
            k, v = (torch.cat([_exact_held(pages[ids].transpose(0, 1).reshape(Hkv, -1, pages.shape[-1])[:, :t], d), x[b, :, None]], 1)
                    for pages, x in ((s["kpages"], knew), (s["vpages"], vnew)))
            for h in range(H):
                x = torch.mv(k[h * Hkv // H], s["q"][b, h].double()) * s["scale"]
                out[b, h] = torch.mv(v[h * Hkv // H].t(), torch.exp(x - torch.logsumexp(x, 0)))
        return out, knew, vnew
    rot = case["rot"]
    pos = torch.cat([torch.arange(h, h + n, dtype=torch.float64) for n, h in zip(lens, _ints(case["held"]))]).to("cuda")
    turn = torch.polar(torch.full((pos.numel(), rot // 2), s["factor"], dtype=torch.float64, device="cuda"),
                       pos[:, None] * s["freqs"].double()[None])[:, None]

    def turned(x, by):
        """Pairs of channels as complex numbers, times `by`."""
        y = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        n = by.shape[0]
        y[:n] = x[:n].detach().double()
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(y[:n, :, first].contiguous(), y[:n, :, second].contiguous()) * by
        y[:n, :, first], y[:n, :, second] = z.real, z.imag
        return y

    outs = (turned(s["q"], turn), turned(s["k"], turn))
    return outs if kind == "rotary" else (*outs, turned(s["dq"], turn.conj()), turned(s["dk"], turn.conj()))
