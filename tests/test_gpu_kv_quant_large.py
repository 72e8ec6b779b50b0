"""A cache of more than 2^30 rows a head, rows handed over for far more positions than it has left."""
import pytest
import torch

from paper_2506_11104_amd import binding as B

pytestmark = pytest.mark.gpu


def test_rows_behind_the_end_of_a_cache_of_2_to_the_30_rows():
    """Start and rows together lie beyond 2^31: what fits is written, nothing else. (One row, repeated: k and v are broadcast.)"""
    cap, d, block, left, n = (1 << 30) + 64, 64, 128, 5, 1 << 30
    c = B.quant_cache(1, 1, cap, d, torch.int8, block)
    c.kscale.fill_(100), c.vscale.fill_(90)
    k, v = ((torch.arange(d, device="cuda") - 30.0 + x)[None, None, None].to(torch.bfloat16).expand(1, 1, n, d) for x in (0, 3))
    B.dam_kv_quantize(c, k, v, start=torch.tensor([cap - left], dtype=torch.int32, device="cuda"))
    ko, vo = B.dam_kv_dequantize(c, rows=left, pos=cap - left)
    torch.cuda.synchronize()
    assert torch.equal(ko, k[:, :, :left]) and torch.equal(vo, v[:, :, :left])
    last = c.kscale.shape[2] - 1
    for scale, was in ((c.kscale, 100), (c.vscale, 90)):
        assert int((scale != was).sum()) == 1 and int(scale[0, 0, last]) != was
    for codes in (c.k, c.v):
        assert not codes[0, 0, :1 << 16].any() and not codes[0, 0, cap - (1 << 16):cap - left].any()
    del c, codes, scale
    torch.cuda.empty_cache()
