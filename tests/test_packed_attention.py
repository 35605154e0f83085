"""Attention over packed sequences against the formulas in 64 bits, with bounds that count its roundings."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2412_19829_amd import binding as gb
from tests import packed_reference as ref

gpu = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


# ---- the reference itself, and refusals (CPU) ------------------------------------------------------

def test_reference_gradients_against_differences():
    gen = torch.Generator().manual_seed(3)
    q, k, v, g = (torch.randn(n, 8, dtype=torch.float64, generator=gen) for n in (5, 7, 7, 5))
    got = ref.sequence(q, k, v, g, 0.7, "f32")
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        for at in [(0, 0), (2, 5), (4, 7)]:
            step, loss = 1e-6, []
            for sign in (1, -1):
                y = x.clone()
                y[at] += sign * step
                args = {"dq": (y, k, v), "dk": (q, y, v), "dv": (q, k, y)}[name]
                loss.append((ref.sequence(*args, None, 0.7, "f32")["out"][0] * g).sum())
            assert abs((loss[0] - loss[1]) / (2 * step) - got[name][0][at]) < 1e-7


A = 1 << 20   # an aligned address that nothing reads: every call below is refused on the host


def fwd(p=None, q=A, k=2 * A, v=3 * A, out=4 * A, rest=0, lse=5 * A, cu_q=6 * A, cu_k=0, n=2, tq=8, tk=8, H=4, Hkv=2, d=64):
    p = p or gb.make_packed_params()
    return gb.lib().gformer_packed_attn_fwd(q, k, v, out, rest, lse, cu_q, cu_k, n, tq, tk, H, Hkv, d, ctypes.byref(p), None)


def bwd(p=None, ws=7 * A, ws_bytes=1 << 20, dq=8 * A, dk=9 * A, dv=10 * A, lse=5 * A, cu_k=0, tq=8, tk=8, dout=11 * A, rest=0):
    p = p or gb.make_packed_params()
    return gb.lib().gformer_packed_attn_bwd(A, 2 * A, 3 * A, 4 * A, rest, lse, dout, dq, dk, dv, 6 * A, cu_k, 2, tq, tk, 4, 2, 64,
                                            ctypes.byref(p), ws, ws_bytes, None)


def wrong(**kw):
    p = gb.make_packed_params()
    for name, val in kw.items():
        setattr(p, name, val if not isinstance(val, tuple) else (ctypes.c_int64 * 2)(*val))
    return p


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), 1), (dict(out=0), 1), (dict(cu_q=0), 1), (dict(k=0), 1), (dict(q=A + 8), 1), (dict(cu_q=A + 2), 1), (dict(out=A), 1),
    (dict(n=-1), 1), (dict(tq=-1), 1), (dict(H=3), 1), (dict(Hkv=0), 1), (dict(H=0), 1), (dict(d=96), 2), (dict(tk=9), 1),
    (dict(p=wrong(struct_size=8)), 1), (dict(p=wrong(dtype=2)), 1), (dict(p=wrong(zero_tail=2)), 1), (dict(p=wrong(softmax_scale=NAN)), 1),
    (dict(p=wrong(softmax_scale=INF)), 1), (dict(p=wrong(q_stride=(60, 64))), 1), (dict(p=wrong(q_stride=(256, -64))), 1),
    (dict(p=wrong(k_stride=(32, 64))), 1), (dict(p=wrong(v_stride=((1 << 20) + 8, 64))), 2), (dict(tq=2 ** 31 - 1, tk=2 ** 31 - 1, H=256), 2),
])
def test_forward_refusals(kw, status):
    assert fwd(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(ws=0), 3), (dict(ws_bytes=16639), 3), (dict(ws=A + 16), 1), (dict(dq=0), 1), (dict(lse=0), 1), (dict(dout=0), 1), (dict(dq=A), 1),
    (dict(dk=9 * A, dv=9 * A), 1), (dict(dv=5 * A), 1), (dict(dk=A + 8), 1), (dict(tk=7), 1), (dict(p=wrong(dk_stride=(8, 64))), 1),
    (dict(rest=8 * A), 1), (dict(rest=12 * A, p=gb.make_packed_params(gb.GF_F32)), 1),
])
def test_backward_refusals(kw, status):
    assert bwd(**kw) == status


def test_empty_calls():
    assert fwd(tq=0, tk=0, q=0, k=0, v=0, out=0, cu_q=0) == gb.GF_OK
    assert bwd(tq=0, tk=0) == gb.GF_OK
    assert gb.gformer_packed_attn_bwd_workspace_bytes(10, 10, 1, 2, 2, 64) == 256   # two numbers a query and head
    # and the sums of either part of the heads
    assert gb.gformer_packed_attn_bwd_workspace_bytes(10, 10, 1, 4, 2, 64) == 512 + 2 * 10 * 2 * 64 * 2 * 4
    assert gb.gformer_packed_attn_bwd_workspace_bytes(10, 10, 1, 4, 3, 64) == 0


def test_binding_refuses_what_it_would_misread():
    t = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError, match="device tensor"):
        gb.gformer_packed_attn_fwd(t, t, t, t, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="broadcast"):
        gb._row_strides("q", t[:, :1].expand(4, 3, 64))
    assert gb._row_strides("q", t[:1].as_strided((1, 2, 64), (0, 64, 1))) == [128, 64]


# ---- GPU -------------------------------------------------------------------------------------------

SHAPES = [
    # lens_q, lens_k (None: the same)
    ([1], None),
    ([3, 1, 2], None),
    ([0, 5, 0], None),
    ([128], None),
    ([127, 129, 64], None),
    ([33, 300, 65], None),
    ([1, 40, 0, 130], [77, 40, 9, 257]),       # queries behind keys that are there already
    ([20, 140, 3], [5, 0, 2]),                 # queries that see nothing
    ([130, 5], [9000, 5]),                     # more levels of tiles than lanes
    ([600], None),                             # long enough for waves on different keys
]


def tensors(lens_q, lens_k, H, Hkv, d, dtype, seed, tail=0, layout="dense"):
    gen = torch.Generator().manual_seed(seed)
    make = lambda n, h: torch.randn(n, h, d, generator=gen).to(ref.TYPES[dtype]).cuda()
    tq, tk = sum(lens_q) + tail, sum(lens_k) + tail
    if layout == "fused" and tq == tk:         # one projection's output
        x = make(tq, H + 2 * Hkv)
        q, k, v = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
    else:
        q, k, v = make(tq, H), make(tk, Hkv), make(tk, Hkv)
        if layout == "heads":                  # [heads, rows, d] in memory
            q, k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
    return q, k, v, make(tq, H)


def cu(lens):
    return torch.tensor(ref.offsets(lens), dtype=torch.int32).cuda()


def run(q, k, v, g, lens_q, lens_k, scale, zero_tail=0, fill=7.0, same=False, rest=False):
    out, dq, dk, dv = (torch.full(x.shape, fill, dtype=q.dtype, device="cuda") for x in (q, q, k, k))
    lse = torch.full((q.shape[1], q.shape[0]), fill, device="cuda")
    rest = torch.full_like(out, fill) if rest and q.dtype == torch.bfloat16 else None
    cq, ck = cu(lens_q), None if same else cu(lens_k)
    gb.gformer_packed_attn_fwd(q, k, v, out, cq, ck, lse=lse, out_rest=rest, softmax_scale=scale, zero_tail=zero_tail)
    gb.gformer_packed_attn_bwd(q, k, v, out, lse, g, dq, dk, dv, cq, ck, out_rest=rest, softmax_scale=scale, zero_tail=zero_tail)
    torch.cuda.synchronize()
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv, "rest": rest}


def compare(got, want, lens_q, lens_k):
    nq, nk = sum(lens_q), sum(lens_k)
    for name, (x, bound) in want.items():
        n = nk if name in ("dk", "dv") else nq
        if name == "lse":
            ref.check(got[name][:, :n], x[:, :n], bound[:, :n], name)
        else:
            ref.check(got[name][:n], x[:n], bound[:n], name)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (6, 2), (4, 1)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_values_and_gradients(dtype, d, H, Hkv, shape):
    lens_q, lens_k = SHAPES[shape]
    same = lens_k is None
    lens_k = lens_q if same else lens_k
    q, k, v, g = tensors(lens_q, lens_k, H, Hkv, d, dtype, 10 * shape + H, layout="fused" if same else "heads")
    got = run(q, k, v, g, lens_q, lens_k, d ** -0.5, same=same)
    compare(got, ref.packed(q, k, v, g, lens_q, lens_k, d ** -0.5, dtype), lens_q, lens_k)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(64, 64), (128, 32), (128, 128)])
@pytest.mark.parametrize("lens_q,lens_k", [([127, 129, 64, 33], None), ([1, 140, 0, 130], [77, 140, 9, 257]), ([20, 240, 3], [5, 0, 200])])
def test_many_heads(dtype, d, H, Hkv, lens_q, lens_k):
    """Enough workgroups for the kernels whose waves share the streamed rows (those above have waves on different ones)."""
    lens_k = lens_k or lens_q
    q, k, v, g = tensors(lens_q, lens_k, H, Hkv, d, dtype, H + d, layout="heads")
    got = run(q, k, v, g, lens_q, lens_k, d ** -0.5, rest=True)
    compare(got, ref.packed(q, k, v, g, lens_q, lens_k, d ** -0.5, dtype), lens_q, lens_k)


@gpu
@pytest.mark.parametrize("lens_q,lens_k", [([600], [600]), ([513, 555], [1100, 400])])
def test_single_precision_in_two_streams(lens_q, lens_k):
    """d = 128, with more workgroups than compute units can hold of four streams each; a key that some rows do not see is no number."""
    q, k, v, g = tensors(lens_q, lens_k, 32, 8, 128, "f32", 71, layout="heads")
    want = ref.packed(q, k, v, g, lens_q, lens_k, 0.1, "f32")
    got = run(q, k, v, g, lens_q, lens_k, 0.1)
    compare(got, want, lens_q, lens_k)
    k, v = k.clone(), v.clone()
    last = lens_k[0] - 1                       # the first sequence's last key: its last query alone sees it
    k[last], v[last] = float("nan"), float("inf")
    bad = run(q, k, v, g, lens_q, lens_k, 0.1)
    rows = [i for i in range(sum(lens_q)) if i != lens_q[0] - 1]
    assert torch.equal(bad["out"][rows], got["out"][rows]) and torch.equal(bad["dq"][rows], got["dq"][rows])
    assert bad["out"][lens_q[0] - 1].isnan().all()


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_what_rounding_takes_from_the_output(d):
    """out + rest is the output before its rounding, up to rest's own; dq and dk then come nearer to the formula's."""
    lens = [200, 70]
    q, k, v, g = tensors(lens, lens, 4, 2, d, "bf16", 15)
    want = ref.packed(q, k, v, g, lens, lens, d ** -0.5, "bf16")
    plain, got = run(q, k, v, g, lens, lens, d ** -0.5), run(q, k, v, g, lens, lens, d ** -0.5, rest=True)
    compare(got, want, lens, lens)
    assert torch.equal(plain["out"], got["out"])
    both = got["out"].double().cpu() + got["rest"].double().cpu()
    # what is left: the weights' rounding, and half a step of rest's, which is half a step of out at most
    ref.check(both, want["out"][0], want["out"][1] - ref.HALF["bf16"] * want["out"][0].abs() * (1 - 2 * ref.HALF["bf16"]), "out + rest")
    for name in ("dq", "dk"):
        off = [(x[name].double().cpu() - want[name][0]).norm() for x in (plain, got)]
        assert off[1] < off[0], name


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(8, 2), (128, 128)])
def test_short_sequences_are_rounded_once(d, H, Hkv):
    """Sequences inside one tile: both parts of the scores' gradients go into dq and dk, so that next to their own rounding, of
    relative error r in the mean, only the weights' rounding in the forward pass is left, which delta sees through the output.
    It puts an error of r sqrt(sum_j p_j^2 dp_j^2) into delta, and of that times p_j into every score's gradient p_j (dp_j - delta):
    with independent values, of r sqrt(sum_j p_j^2) times a row of dq.  Scores of variance 1 have sum_j p_j^2 = e / n for n keys (0.6 for two),
    and rows weigh as much in dq's norm; over rows of 2 to n keys the weighted mean is (0.36 + 7.4 sum 1 / n^2) / (0.6 + 2.7 sum 1 / n),
    sums from 3: 0.44 for n = 32, 0.6 for n = 5.  So dq and dk are off by at most sqrt(1 + 0.6) = 1.27 times one rounding, and by
    sqrt(2) and more with another one."""
    lens = [5, 16, 31, 28, 2, 9, 32]
    q, k, v, g = tensors(lens, lens, H, Hkv, d, "bf16", 51)
    want = ref.packed(q, k, v, g, lens, lens, d ** -0.5, "bf16")
    got = run(q, k, v, g, lens, lens, d ** -0.5, rest=True)
    compare(got, want, lens, lens)
    for name in ("dq", "dk"):
        exact = want[name][0].double()
        off = lambda x: float((x.double().to(exact.device) - exact).norm())
        assert off(got[name]) < 1.27 * off(exact.to(torch.bfloat16)), name


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 1e-42, 1.5])
def test_scales(dtype, scale):
    lens = [70, 200]
    q, k, v, g = tensors(lens, lens, 2, 1, 64, dtype, 5)
    compare(run(q, k, v, g, lens, lens, scale), ref.packed(q, k, v, g, lens, lens, scale, dtype), lens, lens)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_short_sequences(dtype):
    lens = [(7 * i) % 5 for i in range(300)]   # the search for a tile's sequence takes more than one step
    q, k, v, g = tensors(lens, lens, 2, 2, 64, dtype, 6)
    compare(run(q, k, v, g, lens, lens, 0.125), ref.packed(q, k, v, g, lens, lens, 0.125, dtype), lens, lens)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("zero", [0, 1])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (4, 1), (64, 64)])
def test_rows_behind_the_last_sequence(dtype, zero, H, Hkv):
    lens, tail = [5, 130], 300
    q, k, v, g = tensors(lens, lens, H, Hkv, 64, dtype, 7, tail=tail)
    for x in (q, k, v, g):
        x[sum(lens):] = NAN
    got = run(q, k, v, g, lens, lens, 0.125, zero_tail=zero)
    compare(got, ref.packed(q[:135], k[:135], v[:135], g[:135], lens, lens, 0.125, dtype), lens, lens)
    for name in ("out", "dq", "dk", "dv"):
        assert (got[name][sum(lens):] == (0.0 if zero else 7.0)).all(), name
    assert (got["lse"][:, sum(lens):] == 7.0).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad,H,Hkv", [(NAN, 2, 1), (INF, 2, 1), (-INF, 2, 1), (NAN, 96, 96), (INF, 96, 48)])
def test_what_a_row_does_not_see_has_no_part_in_it(dtype, d, bad, H, Hkv):
    # sequence 0: a key and a value that only its later queries see, and a query and a gradient that are no part of what
    # later keys get; sequence 1 sees nothing of either
    lens, at = [150, 90], 70
    q, k, v, g = tensors(lens, lens, H, Hkv, d, dtype, 8)
    clean = ref.packed(q, k, v, g, lens, lens, 0.1, dtype)
    for name, x in (("k", k), ("v", v)):
        kept = x[at].clone()
        x[at] = bad
        got = run(q, k, v, g, lens, lens, 0.1)
        for rows in (slice(0, at), slice(150, 240)):
            for n in ("out", "dq"):
                ref.check(got[n][rows], clean[n][0][rows], clean[n][1][rows], f"{n} with {name} of a later key {bad}")
            ref.check(got["lse"][:, rows], clean["lse"][0][:, rows], clean["lse"][1][:, rows], "lse")
        x[at] = kept
    for name, x in (("q", q), ("g", g)):
        kept = x[at].clone()
        x[at] = bad
        got = run(q, k, v, g, lens, lens, 0.1)
        for rows in (slice(at + 1, 150), slice(150, 240)):
            for n in ("dk", "dv"):
                ref.check(got[n][rows], clean[n][0][rows], clean[n][1][rows], f"{n} with {name} of an earlier query {bad}")
        x[at] = kept


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_that_sees_no_number_is_none(dtype):
    lens = [100]
    q, k, v, g = tensors(lens, lens, 1, 1, 64, dtype, 9)
    v[10] = NAN
    out = run(q, k, v, g, lens, lens, 0.1)["out"]
    assert torch.isnan(out[10:]).all() and not torch.isnan(out[:10]).any()


@gpu
def test_large_scores_and_offsets_out_of_range():
    lens = [64, 200]
    q, k, v, g = tensors(lens, lens, 2, 2, 64, "bf16", 11)
    compare(run(q * 16, k * 16, v, g, lens, lens, 1.0), ref.packed(q * 16, k * 16, v, g, lens, lens, 1.0, "bf16"), lens, lens)
    # offsets past the tensors, or descending: computed on what there is, nothing outside is touched
    out = torch.zeros(264 + 64, 2, 64, dtype=q.dtype, device="cuda")
    for bad in ([0, 64, 5000], [0, 300, 100], [-7, 64, 264]):
        gb.gformer_packed_attn_fwd(q, k, v, out[:264], torch.tensor(bad, dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert (out[264:] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_wrapper(dtype):
    from paper_2412_19829_amd.autograd import gformer_packed_attention
    lens, tail = [90, 1, 140], 20
    q, k, v, g = tensors(lens, lens, 4, 2, 64, dtype, 12, tail=tail)
    want = ref.packed(q, k, v, g, lens, lens, 0.125, dtype)
    leaves = [x.clone().requires_grad_(True) for x in (q, k, v)]
    out = gformer_packed_attention(*leaves, cu(lens), softmax_scale=0.125)
    out.backward(g.transpose(0, 1).contiguous().transpose(0, 1))
    for name, x in zip(("out", "dq", "dk", "dv"), (out, *(t.grad for t in leaves))):
        ref.check(x, *want[name], name)
    # a gradient that is one number broadcast, and views of one fused tensor as leaves
    x = torch.cat([q, k, v], 1).requires_grad_(True)
    gformer_packed_attention(x[:, :4], x[:, 4:6], x[:, 6:], cu(lens), softmax_scale=0.125).float().sum().backward()
    want = ref.packed(q, k, v, torch.ones_like(q) * (torch.arange(251) < 231)[:, None, None].cuda(), lens, lens, 0.125, dtype)
    for name, at in (("dq", slice(0, 4)), ("dk", slice(4, 6)), ("dv", slice(6, 8))):
        ref.check(x.grad[:, at], *want[name], name)


@gpu
def test_captured_and_on_another_stream():
    lens = [300, 41]
    q, k, v, g = tensors(lens, lens, 4, 2, 128, "bf16", 13)
    want = run(q, k, v, g, lens, lens, 0.1)
    out, dq, dk, dv = (torch.empty_like(x) for x in (q, q, k, k))
    lse = torch.empty(4, q.shape[0], device="cuda")
    ws = torch.empty(gb.gformer_packed_attn_bwd_workspace_bytes(341, 341, 2, 4, 2, 128), dtype=torch.uint8, device="cuda")
    offs = cu(lens)

    def step():
        gb.gformer_packed_attn_fwd(q, k, v, out, offs, lse=lse, softmax_scale=0.1)
        gb.gformer_packed_attn_bwd(q, k, v, out, lse, g, dq, dk, dv, offs, softmax_scale=0.1, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for x in (out, dq, dk, dv, lse):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for name, x in zip(("out", "dq", "dk", "dv", "lse"), (out, dq, dk, dv, lse)):
            assert torch.equal(x, want[name]), name     # no atomics: equal calls give equal bits
        run(q, k, v, g, lens, lens, 0.1)


@gpu
def test_the_extension_module_makes_the_plain_calls(monkeypatch):
    """... with the results of the binding's own code, which makes the others."""
    lens = [50, 90]
    q, k, v, g = tensors(lens, lens, 4, 2, 64, "bf16", 14, layout="fused")
    made = []
    quick = gb._quick
    monkeypatch.setattr(gb, "_quick", lambda *a: made.append(quick(*a)) or made[-1])
    got = run(q, k, v, g, lens, lens, 0.2, rest=True)
    assert made == [True, True]
    out = torch.empty_like(q)
    gb.gformer_packed_attn_fwd(q, k, v, out, cu(lens), softmax_scale=1, stream=torch.cuda.current_stream().cuda_stream)
    assert made[2:] == [False]                          # a scale that is no float
    monkeypatch.setattr(gb, "_quick", lambda *a: False)
    again = run(q, k, v, g, lens, lens, 0.2, rest=True)
    for name in got:
        assert torch.equal(got[name], again[name]), name
    with pytest.raises(ValueError, match="q's shape"):
        gb.gformer_packed_attn_fwd(q, k, v, out[:5], cu(lens))
    monkeypatch.setattr(gb, "_quick", quick)
    with pytest.raises(gb.GformerError, match="status 2"):
        gb.gformer_packed_attn_fwd(*(torch.zeros(8, 2, 32, device="cuda") for _ in range(4)), cu([8]))
    with pytest.raises(gb.GformerError, match="status 3"):
        gb.gformer_packed_attn_bwd(q, k, v, q, got["lse"], q, *(torch.empty_like(x) for x in (q, k, v)), cu(lens),
                                   workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_the_tensors_device_is_current_during_the_call(monkeypatch):
    class On:
        device = "cuda:1"
        def get_device(self):
            return 1
    current = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[-1])
    class Guard:
        def __init__(self, device):
            assert device == "cuda:1"
        def __enter__(self):
            current.append(1)
        def __exit__(self, *_):
            current.pop()
    monkeypatch.setattr(torch.cuda, "device", Guard)
    seen = []
    gb._call(lambda *a: seen.append((current[-1], a)) or gb.GF_OK, On(), 5, "x")
    current.append(1)
    gb._call(lambda *a: seen.append((current[-1], a)) or gb.GF_OK, On(), 6, "y")
    assert seen == [(1, ("x", 5)), (1, ("y", 6))] and current == [0, 1]
    with pytest.raises(gb.GformerError, match="status 2"):
        gb._call(lambda *a: 2, On(), 5)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_node_of_the_extension_module_is_the_wrapper(dtype, monkeypatch):
    from paper_2412_19829_amd import autograd
    lens_q, lens_k, tail = [40, 0, 200, 3], [44, 9, 200, 3], 6
    q, k, v, g = tensors(lens_q, lens_k, 4, 2, 64, dtype, 31, tail=tail)
    q = q.transpose(0, 1).contiguous().transpose(0, 1)   # heads slowest
    starts = cu(lens_q), cu(lens_k)
    gradients = [g, g[:1].expand_as(g), g.transpose(0, 1).contiguous().transpose(0, 1), g.transpose(1, 2).contiguous().transpose(1, 2),
                 torch.cat([g.flatten()[:1], g.flatten()])[1:].view_as(g),
                 torch.empty(len(g), (1 << 20) + 8, dtype=g.dtype, device="cuda")[:, :g[0].numel()].view_as(g).copy_(g)]
    taken = []
    made = gb.packed_attention_node

    def results(gradient):
        leaves = [x.detach().requires_grad_(True) for x in (q, k, v)]
        out = autograd.gformer_packed_attention(*leaves, *starts, softmax_scale=0.125)
        return [out.detach(), *torch.autograd.grad(out, leaves, gradient)]

    def node(*a):
        taken.append(made(*a))
        return taken[-1]

    for gradient in gradients:
        with monkeypatch.context() as m:
            m.setattr(gb, "packed_attention_node", node)
            one = results(gradient)
        with monkeypatch.context() as m:
            m.setattr(gb, "packed_attention_node", lambda *a: None)
            two = results(gradient)
        assert taken[-1] is not None and all(torch.equal(a, b) for a, b in zip(one, two))

    leaves = [x.detach().requires_grad_(True) for x in (q, k, v)]
    out = autograd.gformer_packed_attention(*leaves, *starts, softmax_scale=0.125)
    first = torch.autograd.grad(out, leaves, g, create_graph=True)
    with pytest.raises(RuntimeError, match="once"):
        first[0].float().sum().backward()

    # one leaf alone, none, and a leaf changed before the backward pass
    k1 = k.detach().requires_grad_(True)
    again = autograd.gformer_packed_attention(q, k1, v, *starts, softmax_scale=0.125)
    assert torch.equal(torch.autograd.grad(again, k1, g)[0], first[1].detach())
    assert not autograd.gformer_packed_attention(q, k, v, *starts, softmax_scale=0.125).requires_grad
    out = autograd.gformer_packed_attention(q, k1, v, *starts, softmax_scale=0.125)
    with torch.no_grad():
        k1.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(out, k1, g)


@gpu
def test_the_wrapper_refuses():
    from paper_2412_19829_amd.autograd import gformer_packed_attention
    q, k, v, _ = tensors([8], [8], 4, 2, 64, "bf16", 1)
    with pytest.raises(gb.GformerError):
        gformer_packed_attention(q[:, :3], k, v, cu([8]))          # 3 heads over 2
    with pytest.raises(gb.GformerError):
        gformer_packed_attention(q[..., :48], k[..., :48], v[..., :48], cu([8]))
    for bad in ((q, k.float(), v, cu([8])), (q, k, v[:4], cu([8])), (q, k, v, cu([8]).long()), (q.cpu(), k, v, cu([8])),
                (q[:4], k, v, cu([4])), (q, k, v, cu([8]), cu([8, 0])), (q[0], k, v, cu([8]))):
        with pytest.raises((ValueError, gb.GformerError)):
            gformer_packed_attention(*bad)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_training_step(dtype):
    from paper_2412_19829_amd.autograd import gformer_packed_attention
    lens = [70, 1, 200]
    q, k, v, g = tensors(lens, lens, 8, 2, 64, dtype, 41, tail=9)
    offs = cu(lens)
    leaves = [x.clone().requires_grad_(True) for x in (q, k, v)]

    def step():
        out = gformer_packed_attention(*leaves, offs, softmax_scale=0.125)
        return [out.detach(), *torch.autograd.grad(out, leaves, g)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [x.clone() for x in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for i in range(3):
        for x in got:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert all(torch.equal(a, b) for a, b in zip(step(), want)), i   # the program's own, between the replays
    # other values in the same places
    with torch.no_grad():
        for x in leaves:
            x.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, step()))


@gpu
@pytest.mark.parametrize("node", [True, False])
@pytest.mark.parametrize("lens_q,lens_k,tail", [([], [], 0), ([], [], 5), ([0, 0], [0, 0], 0), ([0], [7], 0), ([7], [0], 0), ([0, 3], [4, 0], 2)])
def test_calls_with_nothing_to_do(lens_q, lens_k, tail, node, monkeypatch):
    from paper_2412_19829_amd.autograd import gformer_packed_attention
    if not node:
        monkeypatch.setattr(gb, "packed_attention_node", lambda *a: None)
    q, k, v, g = tensors(lens_q, lens_k, 4, 2, 64, "bf16", 3, tail=tail)
    leaves = [x.requires_grad_(True) for x in (q, k, v)]
    out = gformer_packed_attention(*leaves, cu(lens_q), cu(lens_k))
    grads = torch.autograd.grad(out, leaves, g)
    assert out.shape == q.shape and all(a.shape == b.shape for a, b in zip(grads, leaves))
    assert not out.any() and not any(x.any() for x in grads)


def test_the_backward_workspace_stays_bounded():
    """Parts of the query heads never take more sums than four 128-row workgroups for each of a card's compute units hold."""
    for H, Hkv in ((127, 1), (7, 1), (28, 4), (64, 1), (1024, 1), (48, 2), (16, 16)):
        for total in (1, 100, 5000, 20000, 40000, 1 << 20):
            for d in (64, 128):
                p = gb.make_packed_params()
                sums = gb.gformer_packed_attn_bwd_workspace_bytes(0, total, 1, H, Hkv, d, p)
                assert sums <= 4 * 512 * 128 * d * 8


# The refusals below come before the pointers are looked at, so that a call of the largest size, with a null pointer in it, is
# refused for the pointer.
@pytest.mark.parametrize("dtype,d,few", [(gb.GF_BF16, 64, 512), (gb.GF_BF16, 128, 512), (gb.GF_F32, 64, 512), (gb.GF_F32, 128, 256)])
@pytest.mark.parametrize("H,Hkv", [(32, 32), (32, 8), (5, 1)])
def test_launches_stay_within_what_one_may_have(dtype, d, few, H, Hkv):
    """A launch has less than 2^32 threads; 8 rows of n sequences take n + 1 tiles a head, of 256 threads for queries and of `few` for keys
    (a workgroup for every part of the query heads that share them)."""
    p = gb.make_packed_params(dtype)
    most = (2 ** 32 - 1) // 256 // H - 1
    assert fwd(p=p, q=0, n=most, H=H, Hkv=Hkv, d=d) == gb.GF_ERR_INVALID_ARG
    assert fwd(p=p, q=0, n=most + 1, H=H, Hkv=Hkv, d=d) == gb.GF_ERR_UNSUPPORTED
    need = lambda n: gb.gformer_packed_attn_bwd_workspace_bytes(8, 8, n, H, Hkv, d, p)
    groups = max(1, round((need(1) - 256 * -(-8 * H * 8 // 256)) / (8 * Hkv * d * 8)))   # parts of the query heads, by their sums
    keys = (2 ** 32 - 1) // few // (Hkv * groups) - 1
    assert need(min(most, keys)) > 0 and need(min(most, keys) + 1) == 0
    call = lambda n: gb.lib().gformer_packed_attn_bwd(0, 2 * A, 3 * A, 4 * A, 0, 5 * A, 11 * A, 8 * A, 9 * A, 10 * A, 6 * A, 0, n, 8, 8, H, Hkv, d,
                                                      ctypes.byref(p), 7 * A, 1 << 20, None)
    assert call(min(most, keys)) == gb.GF_ERR_INVALID_ARG and call(min(most, keys) + 1) == gb.GF_ERR_UNSUPPORTED


def test_long_launches_stay_within_what_one_may_have():
    """Long sequences: tiles of 128 rows."""
    p = gb.make_packed_params()
    rows = 1 << 30
    H = ((2 ** 32 - 1) // 256) // (rows // 128 + 2)
    for heads, status in ((H, gb.GF_ERR_INVALID_ARG), (H + 1, gb.GF_ERR_UNSUPPORTED), (2 ** 31 - 1, gb.GF_ERR_UNSUPPORTED)):
        assert fwd(p=p, q=0, n=1, tq=rows, tk=rows, H=heads, Hkv=heads) == status
        assert gb.lib().gformer_packed_attn_bwd(0, 2 * A, 3 * A, 4 * A, 0, 5 * A, 11 * A, 8 * A, 9 * A, 10 * A, 6 * A, 0, 1, rows, rows, heads, heads,
                                                64, ctypes.byref(p), 7 * A, 1 << 20, None) == status


def test_dense_rows_are_as_long_as_strided_ones_may_be():
    """Rows of 2^20 elements at most, whether the strides are named or left to the library."""
    for d in (64, 128):
        heads = (1 << 20) // d
        for h, status in ((heads, gb.GF_ERR_INVALID_ARG), (heads + 1, gb.GF_ERR_UNSUPPORTED), ((1 << 26) // d, gb.GF_ERR_UNSUPPORTED)):
            for p in (wrong(), wrong(**{f"{x}_stride": (h * d, d) for x in ("q", "k", "v", "o")})):
                assert fwd(p=p, q=0, tq=3, tk=3, H=h, Hkv=h, d=d) == status   # where the length is fine, for the null pointer
    p = gb.make_packed_params()
    assert gb.gformer_packed_attn_bwd_workspace_bytes(3, 3, 1, 1 << 14, 1 << 14, 64, p) > 0
    assert gb.gformer_packed_attn_bwd_workspace_bytes(3, 3, 1, (1 << 14) + 1, (1 << 14) + 1, 64, p) == 0


def test_scales_that_overflow_are_refused():
    for x in (3e38, -3e38, NAN, -INF):
        assert fwd(p=wrong(softmax_scale=x)) == bwd(p=wrong(softmax_scale=x), ws=0) == gb.GF_ERR_INVALID_ARG
    for x in (2.0 ** 127, -2.0 ** 127, 0.0, 1e-40):      # refused for the workspace alone
        assert bwd(p=wrong(softmax_scale=x), ws=0) == 3


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H", [2, 96])
def test_small_scales_of_large_scores(dtype, d, H):
    """Powers of two move from the scale to the queries and keys: the same exponents, so the same bits, and gradients
    that are those times a power of two."""
    lens, by = [70, 200], 2.0 ** 57
    q, k, v, g = tensors(lens, lens, H, H, d, dtype, 61)
    want = run(q, k, v, g, lens, lens, 0.125)
    got = run(q * by, k * by, v, g, lens, lens, 0.125 / by / by)
    for name in ("out", "lse", "dv"):
        assert torch.equal(got[name], want[name]), name
    for name in ("dq", "dk"):
        assert torch.equal(got[name].float() * by, want[name].float()), name


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv", [(4, 2), (128, 32)])
@pytest.mark.parametrize("n", [32, 33, 90])
def test_long_sequences_among_many_short_ones(dtype, H, Hkv, n):
    """Up to 32 sequences are taken in order of falling work, more in the tensors' order: tiles behind a sequence's first in both, at
    either end and in the middle, with prompts that go on behind keys and rows behind the last one."""
    lens_q = [(3 * i) % 4 for i in range(n)]
    lens_q[0], lens_q[n // 2], lens_q[n - 2], lens_q[n - 1] = 300, 513, 129, 65
    lens_k = list(lens_q)
    lens_k[1], lens_k[n // 2], lens_k[n // 3], lens_k[n - 2] = 400, 700, 260, 90
    q, k, v, g = tensors(lens_q, lens_k, H, Hkv, 128, dtype, n + H, tail=150)
    for x, rows in ((q, sum(lens_q)), (g, sum(lens_q)), (k, sum(lens_k)), (v, sum(lens_k))):
        x[rows:] = NAN
    got = run(q, k, v, g, lens_q, lens_k, 0.09, zero_tail=1, rest=True)
    nq, nk = sum(lens_q), sum(lens_k)
    compare(got, ref.packed(q[:nq], k[:nk], v[:nk], g[:nq], lens_q, lens_k, 0.09, dtype), lens_q, lens_k)
    for name, rows in (("out", nq), ("dq", nq), ("dk", nk), ("dv", nk)):
        assert not got[name][rows:].any(), name


@gpu
def test_the_largest_launch():
    """One-token sequences, as many as a launch of 32 heads holds (n tiles, n / 128 and 1 for those that straddle, 32 heads, 256 threads): a row
    gives its value, and a value's gradient is its row's.  The next one is refused."""
    H, d, n = 32, 64, 520222
    assert (n + n // 128 + 1) * H * 256 < 2 ** 32 <= (n + 1 + (n + 1) // 128 + 1) * H * 256
    gen = torch.Generator("cuda").manual_seed(81)
    q, k, v, g = (torch.randn(n + 1, H, d, device="cuda", generator=gen, dtype=torch.bfloat16) for _ in range(4))
    out, rest, dq, dk, dv = (torch.full_like(q, 7.0) for _ in range(5))
    lse = torch.empty(H, n, device="cuda")
    starts = torch.arange(n + 2, dtype=torch.int32, device="cuda")
    cut = [x[:n] for x in (q, k, v, out)]
    gb.gformer_packed_attn_fwd(*cut, starts[:n + 1], lse=lse, out_rest=rest[:n], softmax_scale=0.125)
    gb.gformer_packed_attn_bwd(*cut, lse, g[:n], dq[:n], dk[:n], dv[:n], starts[:n + 1], out_rest=rest[:n], softmax_scale=0.125)
    torch.cuda.synchronize()
    assert torch.equal(out[:n], v[:n]) and torch.equal(dv[:n], g[:n])
    # The one weight is exp2(x - m), m the rounding of the same x: 1 but for half a step of x in base 2, which is |score| U of the weight, and
    # exp2's own step.  The product sees it rounded to bf16, 1, the sum as it is: out is v / sum, whose reciprocal, product and
    # difference to v add a step each, and rest rounds what is left
    score = 0.125 * (q[:n].float() * k[:n].float()).sum(-1, keepdim=True).abs()
    assert (rest[:n].float().abs() <= ref.U * (score + 8) * v[:n].float().abs()).all()
    del score
    # a score of 64 products: 68 roundings and the exponent's few, against fp64 on some rows
    at = torch.tensor([0, 1, 77777, n - 2, n - 1], device="cuda")
    s = 0.125 * (q[at].double() * k[at].double()).sum(-1)
    bound = ref.U * (68 * 0.125 * (q[at].double() * k[at].double()).abs().sum(-1) + 8 * s.abs() + 16)
    assert ((lse[:, at].T.double() - s).abs() <= bound).all()
    assert all((x[n:] == 7.0).all() for x in (out, rest, dq, dk, dv))
    with pytest.raises(gb.GformerError, match="status 2"):
        gb.gformer_packed_attn_fwd(q, k, v, out, starts, softmax_scale=0.125)
