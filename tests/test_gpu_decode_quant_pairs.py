"""Lists per head over the 8-bit cache for every number of (sequence, KV head) pairs around the eights that the XCDs take, with one
workgroup a list and with several: every head's result is that of its sequence and KV head alone."""
import numpy as np
import pytest
import torch

from test_gpu_decode_quant import check, heads, make, pick

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("longest", [60, 900])
@pytest.mark.parametrize("Bn,Hkv", [(1, 1), (1, 2), (3, 1), (1, 4), (1, 5), (3, 2), (7, 1), (1, 8), (9, 1), (3, 4), (7, 2), (4, 4), (9, 2), (4, 5), (17, 2)])
def test_any_number_of_pairs(Bn, Hkv, longest):
    rng = np.random.default_rng(91 + Bn)
    G, cap = 3, 1000
    c, q = make(91, "e4m3", "bf16", Bn, G * Hkv, Hkv, 128, cap, 32)
    lists = [pick(rng, cap, rng.integers(0, longest + 1, G * Hkv)) for _ in range(Bn)]
    lists[0][0] = np.arange(longest)
    got = heads(c, q, lists)
    check(got, c, "e4m3", q, lists)
    again = heads(c, q, lists, out=torch.full_like(q, 7.0))
    torch.cuda.synchronize()
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
