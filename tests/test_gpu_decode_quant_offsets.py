"""Rows of the 8-bit cache that lie far from their head's first one, on either side of what 32-bit offsets of rows serve: the same keys
in a small dense cache give the same bits, in every form."""
import numpy as np
import pytest
import torch

from paper_2506_11104_amd import binding as B
from test_gpu_decode_quant import DTYPE, T, i32, u8

pytestmark = pytest.mark.gpu
ROWS, BLOCK, G = 300, 128, 4


def side_by_side(fmt, d, cap, stride, block):
    """[1][1][cap][d] codes of K and V in rows of `stride` bytes that they share."""
    rows = torch.zeros((1, 1, cap, stride), dtype=torch.uint8, device="cuda")
    scales = [torch.zeros((1, 1, -(-cap // block)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    return B.QuantCache(*(rows[..., x * d:x * d + d].view(DTYPE[fmt]) for x in (0, 1)), *scales, block)


# capacity, bytes between rows, first of the rows that are looked at
PLACES = {
    "32-bit offsets from 2^31 on": lambda d: ((1 << 32) // (16 * d) - 2, 16 * d, (1 << 32) // (16 * d) - 512),
    "32-bit offsets around 2^31": lambda d: ((1 << 32) // (16 * d) - 2, 16 * d, (1 << 31) // (16 * d) - 128),
    "offsets around 2^32": lambda d: ((1 << 32) // (16 * d) + 400, 16 * d, (1 << 32) // (16 * d) - 128),
    "2^24 rows and more": lambda d: ((1 << 24) + 400, 2 * d, (1 << 24) - 128),
    "rows 2^24 bytes apart": lambda d: (ROWS, 1 << 24, 0),
}


@pytest.mark.parametrize("place", list(PLACES))
@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "f32", 128), ("e4m3", "f32", 64), ("int8", "bf16", 64)])
def test_keys_far_from_the_first_row(place, fmt, dtype, d):
    cap, stride, base = PLACES[place](d)
    assert base % BLOCK == 0 and base + ROWS <= cap
    g = torch.Generator().manual_seed(49)
    k, v = (torch.randn((1, 1, ROWS, d), generator=g).cuda() for _ in range(2))
    q = torch.randn((1, G, d), generator=g).to(T[dtype]).cuda()
    far, small = side_by_side(fmt, d, cap, stride, BLOCK), B.quant_cache(1, 1, 384, d, DTYPE[fmt], BLOCK)
    for c, at in ((far, base), (small, 0)):
        B.dam_kv_quantize(c, k, v, pos=at)
    keys = np.arange(0, ROWS, 2)
    per, one, mem = i32(np.arange(G + 1) * 40), i32([0, len(keys)]), u8(1 + np.arange(len(keys)) % 15)
    # a plan: 150 diagonals and twenty columns, at the last row
    val = np.concatenate([-1 - np.arange(149, -1, -1), np.arange(20)])
    table = np.zeros((1, ROWS), np.uint8)
    table[0, :150] = 15

    def forms(c, at):
        columns = i32(np.where(val < 0, val, val + at))
        plan = B.Mask(H=G, L=0, S=ROWS, tile_m=128, tile_n=128, kept_ptr=i32([0, len(val)]), kept_idx=columns,
                      kept_member=u8([15] * len(val)), plan_table=u8(table))
        return [*B.dam_sparse_attn_decode_quantized(q, c, per, i32(np.resize(keys, 40 * G) + at), 40, want_lse=True),
                *B.dam_sparse_attn_decode_grouped_quantized(q, c, one, i32(keys + at), mem, len(keys), want_lse=True),
                *B.dam_sparse_attn_decode_patterns_quantized(q, c, plan, at + ROWS - 1, len(val), want_lse=True),
                *B.dam_kv_dequantize(c, rows=ROWS, pos=at)]

    want, got = forms(small, 0), forms(far, base)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    del far
    torch.cuda.empty_cache()
