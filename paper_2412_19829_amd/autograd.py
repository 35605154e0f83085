"""The layer as a differentiable PyTorch operation (gformer_attn_fwd in forward, gformer_attn_bwd in backward), and
attention over packed sequences likewise (gformer_packed_attn_fwd, gformer_packed_attn_bwd).

Plumbing only: tensors are allocated here (PyTorch is used for device memory and streams) and
every arithmetic step runs in the HIP kernels behind the C ABI.  There is no CPU path.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as gb


class _GformerAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, window, n_sparse_heads, phi, softmax_scale, eps, bidirectional):
        out = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device)
        gb.gformer_attn_fwd(q, k, v, out, window, n_sparse_heads, phi=phi, softmax_scale=softmax_scale,
                            eps=eps, bidirectional=bidirectional)
        ctx.save_for_backward(q, k, v)
        ctx.cfg = (int(window), int(n_sparse_heads), int(phi), float(softmax_scale), float(eps),
                   int(bidirectional))
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v = ctx.saved_tensors
        window, n_sparse_heads, phi, softmax_scale, eps, bidirectional = ctx.cfg
        if dout.stride(-1) != 1:
            dout = dout.contiguous()
        # gradients are laid out like the tensors they belong to
        dq, dk, dv = (torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device)
                      for t in (q, k, v))
        gb.gformer_attn_bwd(q, k, v, dout, dq, dk, dv, window, n_sparse_heads, phi=phi,
                            softmax_scale=softmax_scale, eps=eps, bidirectional=bidirectional)
        return dq, dk, dv, None, None, None, None, None, None


def gformer_attention(q, k, v, window: int, n_sparse_heads: int, *, phi=gb.GF_PHI_ELU1,
                      softmax_scale: float = 1.0, eps: float = 0.0, bidirectional: int = 0):
    """GFormer attention on [B, H, N, d] device tensors (bf16 or fp32, any strides with a
    contiguous last dimension): heads [0, n_sparse_heads) windowed softmax, the rest linear.
    Differentiable with respect to q, k and v."""
    return _GformerAttention.apply(q, k, v, window, n_sparse_heads, phi, softmax_scale, eps,
                                   bidirectional)


def _fits(t):
    """Whether a [rows, heads, d] tensor can be handed over as it is; a gradient may come in any layout."""
    return (t.stride(-1) == 1 and t.data_ptr() % 16 == 0 and
            all(n == 1 or (x >= t.shape[-1] and x % 8 == 0) for n, x in zip(t.shape[:2], t.stride()[:2])) and
            (t.shape[0] == 1 or t.stride(0) <= 1 << 20))


class _GformerPackedAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_q, cu_k, softmax_scale):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[1], q.shape[0], dtype=torch.float32, device=q.device)
        rest = torch.empty_like(out) if q.dtype == torch.bfloat16 and any(ctx.needs_input_grad) else None
        gb.gformer_packed_attn_fwd(q, k, v, out, cu_q, cu_k, lse=lse, out_rest=rest, softmax_scale=softmax_scale, zero_tail=1)
        ctx.save_for_backward(q, k, v, out, rest, lse, cu_q, cu_k)
        ctx.softmax_scale = softmax_scale
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, rest, lse, cu_q, cu_k = ctx.saved_tensors
        if not _fits(dout):
            dout = dout.contiguous()
            if not _fits(dout):
                dout = dout.clone(memory_format=torch.contiguous_format)
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        gb.gformer_packed_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, cu_q, cu_k, out_rest=rest,
                                   softmax_scale=ctx.softmax_scale, zero_tail=1)
        return dq, dk, dv, None, None, None


def gformer_packed_attention(q, k, v, cu_q, cu_k=None, *, softmax_scale: float = 1.0):
    """Causal attention over packed sequences: q [total_q, H, d], k, v [total_k, Hkv, d] device tensors (bf16 or fp32, any
    strides with a contiguous last dimension, H a multiple of Hkv), cu_q and cu_k int32 [n_seqs + 1] offsets on the
    device (cu_k=None: the same sequences).  With more keys than queries a sequence's queries are its last; rows
    behind the last sequence give zeros.  Differentiable once with respect to q, k and v.  Both passes can be captured in a graph, as
    long as no eager graph of the same leaves is alive: torch keeps one node a leaf for its gradient, with the stream that it was made on."""
    out = gb.packed_attention_node(q, k, v, cu_q, cu_k, float(softmax_scale))
    return _GformerPackedAttention.apply(q, k, v, cu_q, cu_k, float(softmax_scale)) if out is None else out
