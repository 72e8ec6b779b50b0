"""The softmax weights of merged lists and plans over the 8-bit cache with bf16 queries, seen in outputs near 0: values of either sign
that nearly cancel leave an output whose own rounding is far below an error of the weights.

Every query has one element that is not 0, so a raw logit is exact. With u = 2^-24 and |z| <= 2 in every list: the exponent of a
weight is off by the roundings of the scale in log2 units, of the reference and of their sum, 8 u |z| in all, the exponential by
2 u, so a weight by 18 u; it goes in as two bf16 terms, off by 2^-17 of it. Sums over n keys in fp32, n u of the weights and 2 n u
of the terms' products (exact ones); the merges and the division 10 u. So, A being sum_j p_j |v_j|,
  |dO| <= A (2^-17 + 36 u + (3 n + 10) u) + 2^-8 |O|."""
import numpy as np
import pytest
import torch

from paper_2506_11104_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def cut_off(w):
    """What is left of fp32 numbers after two terms of 8 bits that are cut off, relative to them: up to 2^-15."""
    w = w.astype(np.float32)
    for _ in range(2):
        w = w - (w.view(np.uint32) & 0xFFFF0000).view(np.float32)
    return w


def keys_and_values(rng, q0, scale, d):
    """Codes of four keys' first element and [4][d] values for them: the key of the largest logit and one whose weight has hardly
    any bit beyond the 16th have negative values, two whose weights have many positive ones (so that terms that are cut off would
    err to one side), whose weighted sums are as small as those of 50000 draws get."""
    codes = np.arange(-127, 128)
    z = q0 * codes * scale
    rel = np.exp(z - z.max())
    order = np.argsort(cut_off(rel) / rel)
    top = order[np.argmax(rel[order])]
    order = order[order != top]
    at = np.array([top, order[0], order[-1], order[-2]])
    v = rng.integers(1, 128, (4, 50000)) * np.array([-1, -1, 1, 1])[:, None]
    w = np.exp(z[at])
    return codes[at], v[:, np.argsort(np.abs(w @ v) / (w @ np.abs(v)))[:d]]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", ["merged", "plan"])
def test_weights_are_as_good_as_two_rounded_terms(form, d):
    rng = np.random.default_rng(71)
    Bn, n, block, scale = 40, 4, 16, np.float32(1 / 256)
    c = B.quant_cache(Bn, 1, block, d, torch.int8, block)
    c.kscale.fill_(127), c.vscale.fill_(127)             # codes are the values
    q0 = rng.choice([-1, 1], Bn) * (1 + rng.integers(0, 128, Bn) / 128) * 2
    kcode, v = (np.stack(x) for x in zip(*(keys_and_values(rng, x, float(scale), d) for x in q0)))
    z = q0[:, None] * kcode * float(scale)
    assert np.abs(z).max() <= 2
    w = np.exp(z)
    c.k[:, 0, :n, 0] = torch.from_numpy(kcode.astype(np.int8)).cuda()
    c.v[:, 0, :n] = torch.from_numpy(v.astype(np.int8)).cuda()
    q = torch.zeros((Bn, 1, d), dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = torch.from_numpy(q0).to(torch.bfloat16)
    assert np.array_equal(q[:, 0, 0].double().cpu().numpy(), q0)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    ones = torch.ones(n, dtype=torch.uint8, device="cuda")
    if form == "merged":
        out = B.dam_sparse_attn_decode_grouped_quantized(q, c, i32([0, n]), i32(range(n)), ones, n, scale=float(scale), shared_lists=True)
    else:
        plan = B.Mask(H=1, L=0, S=n, tile_m=128, tile_n=128, kept_ptr=i32([0, n]), kept_idx=i32(range(-n, 0)), kept_member=ones,
                      plan_table=torch.ones((1, n), dtype=torch.uint8, device="cuda"))
        out = B.dam_sparse_attn_decode_patterns_quantized(q, c, plan, n - 1, n, scale=float(scale))
    got, L = out[:, 0].double().cpu().numpy(), w.sum(1)[:, None]
    O, A = np.einsum("bn,bnd->bd", w, v) / L, np.einsum("bn,bnd->bd", w, np.abs(v)) / L
    err = np.abs(got - O) / (A * (2.0 ** -17 + (36 + 3 * n + 10) * U) + 2.0 ** -8 * np.abs(O))
    assert err.max() <= 1, f"{err.max():.2f} of the bound, beyond it in {(err > 1).mean():.1%}"
