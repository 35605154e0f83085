"""The operators of packed prompts and of the paged cache, as a program calls them, beside the same
operators in elementary torch operations.

    own                 False: run() computes the plain form; True: it calls the library
    listed()            the fixed cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program holds before the call (device tensors, page table)
    run(state)          one pass; returns its outputs
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   the same outputs in 64 bits

Four kinds of call:
    prompt  causal attention over packed sequences, and its keys and values written into a paged cache
    train   the same attention with its gradients, through the differentiable wrapper
    decode  one new token of every sequence over the paged cache
    pages   pages of the cache copied to other places (a forked sequence's last page, compaction)
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}


def _prompt(kind, dtype, H, Hkv, d, lens_q, lens_k=None, page=0, tail=0, name=None):
    """lens_q, lens_k: tokens and keys of each sequence, as text; page: tokens a page where the prompt also goes
    into the cache, else 0; tail: rows behind the last sequence, as a batch padded to a fixed size has them."""
    text = lambda v: ",".join(str(int(x)) for x in v)
    c = {"kind": kind, "dtype": dtype, "H": H, "Hkv": Hkv, "d": d, "lens_q": text(lens_q),
         "lens_k": text(lens_q if lens_k is None else lens_k), "page": page, "tail": tail}
    return c if name is None else {"name": name, **c}


def _decode(dtype, H, Hkv, d, lens, page, name=None):
    """lens: tokens of each sequence that are in the cache already, as text."""
    c = {"kind": "decode", "dtype": dtype, "H": H, "Hkv": Hkv, "d": d, "lens": ",".join(str(int(x)) for x in lens),
         "page": page}
    return c if name is None else {"name": name, **c}


def _pages(dtype, Hkv, d, page, pages, copies, name=None):
    c = {"kind": "pages", "dtype": dtype, "Hkv": Hkv, "d": d, "page": page, "pages": pages, "copies": copies}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # One short prompt through a 12-head layer, with its way into the cache: the smallest call, all latency.
        _prompt("prompt", "bf16", 12, 12, 64, [128], page=16, name="prompt_one"),
        # A serving engine's step: whole prompts, chunks that continue one, a single token, a sequence with nothing new.
        _prompt("prompt", "bf16", 32, 8, 128,
                [1531, 512, 77, 1, 2048, 300, 0, 640, 129, 1024, 33, 911],
                [1531, 2048, 77, 1700, 2048, 1213, 50, 640, 1301, 1024, 33, 2047], name="prompts_ragged"),
        # One long prompt of the 32-head model with shared key heads, into pages of 64: the largest forward pass.
        _prompt("prompt", "bf16", 32, 8, 128, [8192], page=64, name="prompt_long"),
        # A training step over packed documents of odd lengths, 16 heads of 64 (the paper's shape), padded to 8192 rows.
        _prompt("train", "bf16", 16, 16, 64, [2048, 513, 1777, 96, 1, 1200, 2001, 300], tail=256, name="train_packed"),
        # A training step of the 32-head model with shared key heads.
        _prompt("train", "bf16", 32, 8, 128, [4096, 3001, 1095], name="train_grouped"),
        # A training step in full precision, 12 heads of 64.
        _prompt("train", "f32", 12, 12, 64, [1024, 300, 700], name="train_f32"),
        # One token for one user of a 12-head model: latency.
        _decode("bf16", 12, 12, 64, [2047], 16, name="decode_one"),
        # One token for a batch of users whose contexts differ, grouped heads.
        _decode("bf16", 32, 8, 128,
                [8191, 4096, 77, 1300, 2500, 6000, 1, 0, 3333, 511, 512, 7100, 900, 4800, 64, 2222,
                 5000, 127, 128, 6789, 1024, 3100, 40, 8000, 1999, 700, 4321, 260, 7777, 15, 5555, 1600],
                64, name="decode_batch"),
        # A few users with very long contexts: the cache's length is what there is to split.
        _decode("bf16", 32, 8, 128, [32767, 32768, 20000, 31111], 128, name="decode_long"),
        # Full precision, every head with keys of its own.
        _decode("f32", 16, 16, 64, [2048, 1000, 3000, 17, 4095, 1], 32, name="decode_f32"),
        # Forked sequences take copies of their last, partly filled pages.
        _pages("bf16", 8, 128, 64, 512, 16, name="pages_fork"),
        # Compaction: the pages at the cache's end move into the holes in front of them.
        _pages("bf16", 8, 128, 64, 4096, 1024, name="pages_compact"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# what a drawn case may cost, and how many padded scores the plain form may hold
_LARGEST = {"prompt": "prompt_long", "train": "train_grouped", "decode": "decode_long", "pages": "pages_compact"}
_MOST_SCORES = 32 * 8192 * 8192


def _heads(rng):
    H = rng.choice([8, 12, 16, 32])
    return H, rng.choice([x for x in (1, 2, 4, 8, H) if H % x == 0])


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "train", "train", "decode", "decode", "decode", "pages"])
    d = rng.choice([64, 128])
    top = next(work(c) for c in listed() if c["name"] == _LARGEST[kind])
    if kind == "pages":
        page = rng.choice([16, 32, 64, 128])
        while True:
            pages = _log_int(rng, 64, 4096)
            case = _pages(rng.choice(["bf16", "f32"]), rng.choice([1, 2, 4, 8, 12]), d, page, pages,
                          _log_int(rng, 1, pages // 2))
            if work(case)["bytes"] <= top["bytes"] and pages * page <= 4096 * 64:
                return case
    H, Hkv = _heads(rng)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "decode":
        B, longest = _log_int(rng, 1, 48), _log_int(rng, 16, 32768)
        while True:
            case = _decode(dtype, H, Hkv, d, [rng.choice([longest, rng.randint(0, longest)]) for _ in range(B)],
                           rng.choice([16, 32, 64, 128, 256]))
            if all(work(case)[x] <= top[x] for x in top):
                return case
            B, longest = max(1, B // 2), max(1, longest * 2 // 3)
    n, longest = _log_int(rng, 1, 16), _log_int(rng, 16, 8192 if dtype == "bf16" else 2048)
    page = rng.choice([0, 16, 64]) if kind == "prompt" else 0
    continues = kind == "prompt" and page == 0 and rng.random() < 0.5
    tail = rng.choice([0, 0, rng.randint(1, 200)])
    while True:
        lens_q = [longest] + [rng.randint(1, longest) for _ in range(n - 1)]
        lens_k = [x + rng.randint(0, longest) * rng.randint(0, 1) for x in lens_q] if continues else lens_q
        case = _prompt(kind, dtype, H, Hkv, d, lens_q, lens_k, page=page, tail=tail)
        # what 32 bits cost over 16: the rate of products in single precision is a sixteenth
        need = {x: v * (16 if dtype == "f32" and x == "flops" else 1) for x, v in work(case).items()}
        if all(need[x] <= top[x] for x in top) and n * H * max(lens_q) * max(lens_k) <= _MOST_SCORES:
            return case
        n, longest = (n // 2, longest) if n > 1 else (n, longest * 2 // 3)


# ---- inputs --------------------------------------------------------------------------------
def _ints(text):
    return [int(x) for x in text.split(",")]


def _offsets(lens, device):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device=device)


def _table(gen, lens, page, spare):
    """A page table for sequences of up to `lens` tokens: every page anywhere in the cache, each used once."""
    need = [-(-x // page) for x in lens]
    pages = sum(need) + spare
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    width = max(max(need), 1)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dt, d, kind = DTYPES[case["dtype"]], case["d"], case["kind"]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(dt)

    s = dict(case, scale=1.0 / math.sqrt(d))
    if kind == "pages":
        # copies read pages of the cache's second half and write pages of its first: none is both
        half = case["pages"] // 2
        s["src"] = (half + torch.randperm(case["pages"] - half, device="cuda", generator=gen)[:case["copies"]]).to(torch.int32)
        s["dst"] = torch.randperm(half, device="cuda", generator=gen)[:case["copies"]].to(torch.int32)
        s["kpages"], s["vpages"] = (normal(case["pages"], case["Hkv"], case["page"], d) for _ in range(2))
        return s
    H, Hkv = case["H"], case["Hkv"]
    if kind == "decode":
        lens = _ints(case["lens"])
        s["B"], s["longest"] = len(lens), max(lens)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["table"], pages = _table(gen, [x + 1 for x in lens], case["page"], 3)
        s["kpages"], s["vpages"] = (normal(pages, Hkv, case["page"], d) for _ in range(2))
        s["q"], s["k"], s["v"] = normal(len(lens), H, d), normal(len(lens), Hkv, d), normal(len(lens), Hkv, d)
        s["out"] = torch.empty_like(s["q"])
        return s
    lens_q, lens_k = _ints(case["lens_q"]), _ints(case["lens_k"])
    s["longest_q"], s["longest_k"] = max(lens_q), max(lens_k)
    s["cu_q"], s["cu_k"] = _offsets(lens_q, "cuda"), _offsets(lens_k, "cuda")
    tq, tk = sum(lens_q) + case["tail"], sum(lens_k) + case["tail"]
    # one fused projection's output where the sequences are the same, as a layer has it
    if case["lens_q"] == case["lens_k"]:
        qkv = normal(tq, H + 2 * Hkv, d)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    else:
        s["q"], s["k"], s["v"] = normal(tq, H, d), normal(tk, Hkv, d), normal(tk, Hkv, d)
    if kind == "train":
        s["q"], s["k"], s["v"] = (x.contiguous().requires_grad_(True) for x in (s["q"], s["k"], s["v"]))
        s["dout"] = normal(tq, H, d)
        s["dout"][sum(lens_q):] = 0        # rows that pad the batch have no gradient
    else:
        s["out"] = torch.zeros(tq, H, d, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(H, tq, dtype=torch.float32, device="cuda")
    if case["page"]:
        s["table"], pages = _table(gen, lens_k, case["page"], 3)
        s["start"] = torch.zeros(len(lens_k), dtype=torch.int32, device="cuda")
        s["kpages"], s["vpages"] = (torch.zeros(pages, Hkv, case["page"], d, dtype=dt, device="cuda") for _ in range(2))
    return s


# ---- the plain forms -----------------------------------------------------------------------
def _places(cu, rows):
    """(sequence, position, in one) of every row of a packed tensor."""
    row = torch.arange(rows, device=cu.device)
    seq = torch.searchsorted(cu[1:].long(), row, right=True)
    inside = seq < cu.numel() - 1
    seq = seq.clamp(max=cu.numel() - 2)
    return seq, torch.where(inside, row - cu.long()[seq], 0), inside


def _padded(x, seq, pos, inside, n, longest):
    """[rows, heads, d] -> [n, heads, longest, d] in 32 bits, with zeros where a sequence has ended."""
    out = torch.zeros(n, longest, *x.shape[1:], device=x.device)
    return out.index_put((seq[inside], pos[inside]), x[inside].float()).transpose(1, 2)


def _plain_attention(q, k, v, cu_q, cu_k, longest_q, longest_k, scale):
    n, H, Hkv, d = cu_q.numel() - 1, q.shape[1], k.shape[1], q.shape[2]
    sq, sk = _places(cu_q, q.shape[0]), _places(cu_k, k.shape[0])
    pq = _padded(q, *sq, n, longest_q).reshape(n, Hkv, H // Hkv * longest_q, d)
    pk, pv = _padded(k, *sk, n, longest_k), _padded(v, *sk, n, longest_k)
    scores = (pq @ pk.transpose(-1, -2)).view(n, Hkv, H // Hkv, longest_q, longest_k) * scale
    nq, nk = (cu_q[1:] - cu_q[:-1]).long(), (cu_k[1:] - cu_k[:-1]).long()
    i, j = torch.arange(longest_q, device=q.device), torch.arange(longest_k, device=q.device)
    hidden = (j[None, None] > (i[None, :] + (nk - nq)[:, None])[:, :, None]) | (j[None, None] >= nk[:, None, None])
    scores = scores.masked_fill(hidden[:, None, None], -math.inf)
    top = scores.detach().amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (scores - top).exp()
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    out = (p.view(n, Hkv, -1, longest_k) @ pv).view(n, H, longest_q, d).transpose(1, 2)
    lse = (top + total.log()).view(n, H, longest_q).transpose(1, 2)
    rows = torch.where(sq[2][:, None, None], out[sq[0], sq[1]], 0.0)
    return rows.to(q.dtype), torch.where(sq[2][:, None], lse[sq[0], sq[1]], 0.0).t()


def _plain_fill(x, pages, table, start, cu, page):
    seq, pos, inside = _places(cu, x.shape[0])
    seq, pos = seq[inside], pos[inside] + start.long()[seq[inside]]
    pages[table[seq, pos // page].long(), :, pos % page] = x[inside]


def _plain_decode(s):
    B, H, Hkv, d, page = s["B"], s["H"], s["Hkv"], s["d"], s["page"]
    t, users = s["lens"].long(), torch.arange(s["B"], device="cuda")
    at = s["table"][users, t // page].long()
    s["kpages"][at, :, t % page] = s["k"]
    s["vpages"][at, :, t % page] = s["v"]
    width = s["table"].shape[1]
    rows = s["table"].clamp(min=0).long()
    k, v = (x[rows].transpose(1, 2).reshape(B, Hkv, width * page, d).float() for x in (s["kpages"], s["vpages"]))
    q = s["q"].float().view(B, Hkv, H // Hkv, d)
    hidden = torch.arange(width * page, device="cuda")[None] > t[:, None]
    scores = ((q @ k.transpose(-1, -2)) * s["scale"]).masked_fill(hidden[:, None, None], -math.inf)
    p = (scores - scores.amax(-1, keepdim=True)).exp()
    out = (p / p.sum(-1, keepdim=True)) @ v.masked_fill(hidden[:, None, :, None], 0.0)
    return out.view(B, H, d).to(s["q"].dtype)


def run(s):
    kind = s["kind"]
    if kind == "pages":
        if own:
            from paper_2412_19829_amd import binding as gb
            gb.gformer_pages_copy(s["kpages"], s["vpages"], s["src"], s["dst"])
        else:
            for pages in (s["kpages"], s["vpages"]):
                pages[s["dst"].long()] = pages[s["src"].long()]
        return s["kpages"], s["vpages"]
    if kind == "decode":
        if own:
            from paper_2412_19829_amd import binding as gb
            out = gb.gformer_paged_decode(s["q"], s["k"], s["v"], s["out"], s["kpages"], s["vpages"], s["table"], s["lens"],
                                          max_len=s["longest"] + 1, softmax_scale=s["scale"])
        else:
            out = _plain_decode(s)
        return out, s["kpages"], s["vpages"]
    if kind == "train":
        if own:
            from paper_2412_19829_amd.autograd import gformer_packed_attention
            out = gformer_packed_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], softmax_scale=s["scale"])
        else:
            out, _ = _plain_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["longest_q"], s["longest_k"], s["scale"])
        return (out.detach(), *torch.autograd.grad(out, (s["q"], s["k"], s["v"]), s["dout"]))
    if own:
        from paper_2412_19829_amd import binding as gb
        out, lse = gb.gformer_packed_attn_fwd(s["q"], s["k"], s["v"], s["out"], s["cu_q"], s["cu_k"], lse=s["lse"],
                                              softmax_scale=s["scale"]), s["lse"]
        if s["page"]:
            gb.gformer_paged_fill(s["k"], s["v"], s["kpages"], s["vpages"], s["table"], s["start"], s["cu_k"])
    else:
        out, lse = _plain_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["longest_q"], s["longest_k"], s["scale"])
        if s["page"]:
            _plain_fill(s["k"], s["kpages"], s["table"], s["start"], s["cu_k"], s["page"])
            _plain_fill(s["v"], s["vpages"], s["table"], s["start"], s["cu_k"], s["page"])
    return (out, lse) + ((s["kpages"], s["vpages"]) if s["page"] else ())


# ---- what a pass cannot do without ----------------------------------------------------------
def work(case):
    size, d = BYTES[case["dtype"]], case["d"]
    if case["kind"] == "pages":
        moved = 2 * case["copies"] * case["Hkv"] * case["page"] * d * size     # keys and values
        return {"bytes": 2 * moved + 8 * case["copies"], "flops": 0}
    H, Hkv = case["H"], case["Hkv"]
    if case["kind"] == "decode":
        lens = _ints(case["lens"])
        seen = sum(x + 1 for x in lens)
        # cached keys and values, the new token's in and into its slot, queries in and results out, the pages' numbers
        rows = 2 * (seen - len(lens)) * Hkv + 4 * len(lens) * Hkv + 2 * len(lens) * H
        return {"bytes": rows * d * size + 4 * sum(-(-(x + 1) // case["page"]) + 1 for x in lens), "flops": 4 * seen * H * d}
    lens_q, lens_k = _ints(case["lens_q"]), _ints(case["lens_k"])
    tq, tk = sum(lens_q), sum(lens_k)
    pairs = sum(sum(min(nk, max(0, nk - nq + 1 + i)) for i in range(nq)) for nq, nk in zip(lens_q, lens_k))
    if case["kind"] == "train":
        # q, k, v, dout in, out, dq, dk, dv out; the two products forward and five more backward
        return {"bytes": (4 * tq * H + 4 * tk * Hkv) * d * size, "flops": 14 * pairs * H * d}
    rows = 2 * tq * H + 2 * tk * Hkv + (2 * tk * Hkv if case["page"] else 0)
    return {"bytes": rows * d * size + 4 * tq * H, "flops": 4 * pairs * H * d}


# ---- the same in 64 bits --------------------------------------------------------------------
def _exact_sequence(q, k, v, dout, scale):
    """One sequence's heads, one after another: out, lse and, where dout is given, the three gradients."""
    nq, H, d = q.shape
    nk, group = k.shape[0], H // k.shape[1]
    out, lse = torch.zeros(nq, H, d, dtype=torch.float64, device=q.device), torch.zeros(H, nq, dtype=torch.float64, device=q.device)
    dq, dk, dv = torch.zeros_like(out), torch.zeros(k.shape, dtype=torch.float64, device=q.device), torch.zeros(k.shape, dtype=torch.float64, device=q.device)
    sees = torch.ones(nq, nk, dtype=torch.bool, device=q.device).tril(nk - nq)
    for h in range(H):
        qh, kh, vh = q[:, h].double(), k[:, h // group].double(), v[:, h // group].double()
        x = torch.where(sees, torch.mm(qh, kh.t()) * scale, -math.inf)
        lse[h] = torch.logsumexp(x, 1)
        w = torch.where(sees, torch.exp(x - lse[h][:, None]), 0.0)
        out[:, h] = torch.mm(w, vh)
        if dout is not None:
            g = dout[:, h].double()
            dv[:, h // group] += torch.mm(w.t(), g)
            t = torch.mm(g, vh.t())
            t = w * (t - (w * t).sum(1, keepdim=True)) * scale
            dq[:, h] = torch.mm(t, kh)
            dk[:, h // group] += torch.mm(t.t(), qh)
    return out, lse, dq, dk, dv


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "pages":
        k, v = s["kpages"].double(), s["vpages"].double()
        for i, o in zip(s["src"].tolist(), s["dst"].tolist()):
            k[o], v[o] = k[i], v[i]
        return k, v
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    if case["kind"] == "decode":
        out = torch.zeros(s["B"], H, d, dtype=torch.float64, device="cuda")
        k, v = s["kpages"].double(), s["vpages"].double()
        for b, t in enumerate(_ints(case["lens"])):
            pages = s["table"][b, :t // case["page"] + 1].tolist()
            k[pages[-1], :, t % case["page"]] = s["k"][b].double()
            v[pages[-1], :, t % case["page"]] = s["v"][b].double()
            kb, vb = (x[pages].permute(1, 0, 2, 3).reshape(Hkv, -1, d)[:, :t + 1] for x in (k, v))
            for h in range(H):
                x = torch.mv(kb[h * Hkv // H], s["q"][b, h].double()) * s["scale"]
                out[b, h] = torch.mv(vb[h * Hkv // H].t(), torch.exp(x - torch.logsumexp(x, 0)))
        return out, k, v
    q, k, v = (s[x].detach() for x in "qkv")
    lens_q, lens_k = _ints(case["lens_q"]), _ints(case["lens_k"])
    full = lambda like: torch.zeros(like.shape, dtype=torch.float64, device="cuda")
    out, lse, dq, dk, dv = full(q), torch.zeros(H, q.shape[0], dtype=torch.float64, device="cuda"), full(q), full(k), full(v)
    a = c = 0
    for nq, nk in zip(lens_q, lens_k):
        at, ct = slice(a, a + nq), slice(c, c + nk)
        dout = s["dout"][at] if case["kind"] == "train" else None
        out[at], lse[:, at], dq[at], dk[ct], dv[ct] = _exact_sequence(q[at], k[ct], v[ct], dout, s["scale"])
        a, c = a + nq, c + nk
    if case["kind"] == "train":
        return out, dq, dk, dv
    if not case["page"]:
        return out, lse
    kp, vp, page = s["kpages"].double(), s["vpages"].double(), case["page"]
    c = 0
    for b, n in enumerate(lens_k):
        for first in range(0, n, page):
            m, to = min(page, n - first), int(s["table"][b, first // page])
            kp[to, :, :m] = k[c + first:c + first + m].transpose(0, 1).double()
            vp[to, :, :m] = v[c + first:c + first + m].transpose(0, 1).double()
        c += n
    return out, lse, kp, vp
