"""What gformer_paged_decode_q4 asks for, against its rule written apart: a row of sums and two statistics for every head, for each of the shares and
once more for each sequence, where a sequence may be cut (more than 128 tokens) and there is more than one share."""
from __future__ import annotations

import pytest

from paper_2412_19829_amd import binding as gb


def asked(bf16, B, H, Hkv, d, longest):
    blocks = max(1, (longest + 127) // 128)
    heads, sets = (4 if d == 128 else 8), 1
    if bf16 and d == 128 and H // Hkv > 4 and Hkv * -(-(H // Hkv) // 8) * B * blocks >= 512:
        sets = 2
    at_once = ({64: 4, 128: 4 - sets} if bf16 else {64: 3, 128: 2})[d]                # workgroups of a compute unit
    shares = max(1, min(256 * at_once // (Hkv * -(-(H // Hkv) // (sets * heads))), B * (2 + blocks)))
    if longest <= 128 or shares == 1:
        return 0
    return -(-(shares + B) * H * (d + 2) * 4 // 256) * 256


@pytest.mark.parametrize("longest", [1, 128, 129, 2048, 100001, 1 << 20, (1 << 30) - 1, 1 << 30])
@pytest.mark.parametrize("H,Hkv,d", [(1, 1, 64), (12, 12, 64), (32, 8, 64), (64, 1, 64), (1, 1, 128), (32, 8, 128), (32, 4, 128), (64, 1, 128), (2048, 1024, 128)])
def test_size(H, Hkv, d, longest):
    for bf16 in (True, False):
        p = gb.make_paged_params(gb.GF_BF16 if bf16 else gb.GF_F32)
        for B in (1, 3, 64, 4096, 1 << 20):
            got = gb.gformer_paged_decode_q4_workspace_bytes(B, H, Hkv, d, longest, p)
            assert got == asked(bf16, B, H, Hkv, d, longest), (bf16, B)
