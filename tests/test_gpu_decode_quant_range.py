"""Decodes over the 8-bit cache whose values of V lie anywhere in the format's range, from below 2^-120 to nearly 2^128, in every form.

Tolerances are those of test_gpu_decode_quant.py, with u, n, A, Z and dw as there. In the place of its n 2^-126 (max |v| + 448): a
product of a weight and a scale that is below 2^-126 may be lost, a code of at most 448 (two terms: twice) multiplies it, and
where the list holds a scale of 2^64 or more that border is 2^-82; an output below 2^-126 may be 0. Where sums of
different range meet, a partial result is multiplied by a power of two that is not whole (an exponential and two roundings, and
the rounding of its exponent, a number up to |z| log2 e: 8 u + 4 u Z), and one below 2^-46 of the others may be lost (n 2^-46):
A (16 u + 8 u Z) more for O, 8 u + 4 u Z for lse, n being below 2^16."""
import numpy as np
import pytest
import torch

import oracle
from oracle import quant as oq
from paper_2506_11104_amd import binding as B
from test_gpu_decode_quant import DTYPE, T, U, cache_values, heads, i32, merged, u8

pytestmark = pytest.mark.gpu
SIZES = {"tiny": 2.0 ** -123, "small": 2.0 ** -80, "middle": 1.0, "large": 2.0 ** 75, "huge": 3.3e38}
FORMS = [("e4m3", "bf16", 128), ("int8", "bf16", 128), ("int8", "f32", 64), ("e4m3", "f32", 128), ("e4m3", "bf16", 64)]


def check(got, c, fmt, q, lists):
    out, lse = (x.double().cpu().numpy() for x in got)
    K, V = cache_values(c, fmt)
    qh = q.double().cpu().numpy()
    d, G = qh.shape[2], qh.shape[1] // K.shape[1]
    bf16 = q.dtype == torch.bfloat16
    for b in range(len(lists)):
        for h, keys in enumerate(lists[b]):
            O, L, A, Z = oq.attend(qh[b, h], K[b, h // G], V[b, h // G], keys)
            n, where = len(keys), f"sequence {b} head {h}, {len(keys)} keys"
            if n == 0:
                assert (out[b, h] == 0).all() and lse[b, h] == -np.inf, where
                continue
            assert np.isfinite(out[b, h]).all() and np.isfinite(lse[b, h]), where
            scale = 2.0 ** (c.vscale[b, h // G].cpu().numpy()[keys // c.block].max() - 127.0)
            dw = (2 * d + 16) * U * Z + 4 * U
            tol = A * (2 * dw + 2 * (n + 64) * U + (2.0 ** -16 if bf16 else 0) + (16 + 8 * Z) * U) + (2.0 ** -8 if bf16 else U) * np.abs(O)
            tol = tol + n * 2 * 448 * (2.0 ** -82 if scale >= 2.0 ** 64 else 2.0 ** -126 if scale >= 2.0 ** -64 else 2.0 ** -162) + 2.0 ** -126
            err = np.abs(out[b, h] - O)
            assert (err <= tol).all(), f"{where}: {np.nanmax(err / tol):.2f} of the bound"
            assert abs(lse[b, h] - L) <= (d + 4) * U * Z + dw + (n + 64) * U + (8 + 4 * Z) * U + 2.0 ** -22 * (1 + abs(L)), where


def planned(c, q, lists):
    """The same lists as a plan of columns, at the last position."""
    G, cap = q.shape[1] // c.k.shape[1], c.k.shape[2]
    vflag = np.zeros((q.shape[1], cap), np.uint8)
    for h, keys in enumerate(lists[0]):
        vflag[h, keys] = 1
    ptr, val, mem, table = oracle.pattern_plan(np.zeros_like(vflag), vflag, G)
    plan = B.Mask(H=q.shape[1], L=0, S=cap, tile_m=128, tile_n=128, kept_ptr=i32(ptr), kept_idx=i32(val), kept_member=u8(mem),
                  plan_table=u8(table))
    return B.dam_sparse_attn_decode_patterns_quantized(q, c, plan, cap - 1, int(np.diff(ptr).max()), want_lse=True)


def all_forms(c, fmt, q, lists):
    for f in (heads, merged, planned):
        check(f(c, q, lists), c, fmt, q, lists)


def cache(g, fmt, d, block, sizes, k):
    """sizes: [cap] magnitudes of V's rows."""
    cap = len(sizes)
    c = B.quant_cache(1, 1, cap, d, DTYPE[fmt], block)
    v = (2 * torch.rand((1, 1, cap, d), generator=g, dtype=torch.float64) - 1) * torch.from_numpy(sizes)[:, None]
    B.dam_kv_quantize(c, k.float().cuda(), v.float().cuda())
    return c


@pytest.mark.parametrize("fmt,dtype,d", FORMS)
@pytest.mark.parametrize("cap,order", [(1024, "shuffled"), (1024, "rising"), (1024, "falling"), (9000, "shuffled")])
def test_heads_that_keep_rows_of_some_sizes(fmt, dtype, d, cap, order):
    """Eight heads of one list, each with rows of its own sizes: none is disturbed by what the others keep."""
    rng, block = np.random.default_rng(81), 16
    g = torch.Generator().manual_seed(81)
    names = np.array(list(SIZES))
    of = np.repeat(rng.integers(0, 5, -(-cap // block)), block)[:cap]       # size of a row: its block's
    if order != "shuffled":
        of = np.sort(of) if order == "rising" else -np.sort(-of)
    c = cache(g, fmt, d, block, np.array([SIZES[x] for x in names])[of], torch.randn((1, 1, cap, d), generator=g))
    q = torch.randn((1, 8, d), generator=g).to(T[dtype]).cuda()
    rows = lambda *sizes: np.flatnonzero(np.isin(names[of], sizes))  # noqa: E731
    one_huge = np.sort(np.concatenate([rows("middle"), rows("huge")[:1]]))
    lists = [[rows("tiny"), rows("huge"), np.arange(cap), one_huge, rows("tiny", "small"), rows("small", "middle"),
              rows("tiny")[:0], rows("middle", "large")]]
    all_forms(c, fmt, q, lists)


@pytest.mark.parametrize("fmt,dtype,d", FORMS)
@pytest.mark.parametrize("size", list(SIZES))
def test_logits_that_rise_or_are_all_alike(fmt, dtype, d, size):
    """Each block's largest logit a little above the last one's, so that weights stand above their reference; and all of them 0."""
    cap = 700
    g = torch.Generator().manual_seed(82)
    q = torch.randn((1, 1, d), generator=g).to(T[dtype])
    k = q.float()[:, :, None] / q.float().norm() * torch.arange(cap)[:, None] * 0.02 * d ** 0.5
    c = cache(g, fmt, d, 32, np.full(cap, SIZES[size]), k)
    lists = [[np.arange(cap), np.arange(100, 131), np.arange(cap - 1, cap)]]
    all_forms(c, fmt, q.expand(1, 3, d).contiguous().cuda(), lists)
    all_forms(c, fmt, torch.zeros((1, 3, d), dtype=T[dtype], device="cuda"), lists)


@pytest.mark.parametrize("fmt,dtype,d", FORMS)
def test_a_row_of_another_size_that_the_softmax_drops_or_prefers(fmt, dtype, d):
    """One row far larger, or smaller, than the others, whose logit stands far below or above theirs; rows of zeros beside it."""
    cap, block = 320, 16
    g = torch.Generator().manual_seed(83)
    q = torch.randn((1, 3, d), generator=g).to(T[dtype])
    for a, b in (("huge", "middle"), ("middle", "tiny"), ("tiny", "middle"), ("middle", "huge"), ("huge", "tiny"), ("tiny", "huge")):
        for z in (-30.0, 30.0):
            for at in (0, 170, 319):
                sizes = np.full(cap, SIZES[b])
                sizes[at // block * block:(at // block + 1) * block] = 0
                sizes[at] = SIZES[a]
                k = 0.1 * torch.randn((1, 1, cap, d), generator=g)
                k[0, 0, at] = q[0, 0].float() * z * d ** 0.5 / q[0, 0].float().square().sum()
                c = cache(g, fmt, d, block, sizes, k)
                all_forms(c, fmt, q[:, :1].expand(1, 3, d).contiguous().cuda(), [[np.arange(cap), np.arange(0, cap, 3), np.arange(at, at + 1)]])


@pytest.mark.parametrize("seed", range(16))
def test_scales_of_any_size(seed):
    """Caches whose blocks' scale bytes of V are drawn from all that the library writes, or from some of them, codes at random."""
    rng = np.random.default_rng(8400 + seed)
    fmt, dtype, d = FORMS[seed % len(FORMS)]
    Bn, Hkv, G, block = int(rng.integers(1, 4)), int(rng.integers(1, 4)), int(rng.integers(1, 9)), int(rng.choice([16, 32, 64, 128]))
    cap = int(rng.choice([1, 40, 333, 1500, 6000]))
    c = B.quant_cache(Bn, Hkv, cap, d, DTYPE[fmt], block)
    shape = c.kscale.shape
    pool = (np.arange(250), np.array([0, 1, 120, 249]), np.array([1, 62, 63, 190, 191]), np.array([0, 126, 127, 128]))[seed // 4]
    c.vscale.copy_(torch.from_numpy(rng.choice(pool, shape).astype(np.uint8)))
    c.kscale.copy_(torch.from_numpy(rng.integers(112, 120, shape).astype(np.uint8)))
    for x in (c.k, c.v):  # e4m3 codes up to 0x6F (120) and int8 ones up to 63: less than 2^128 with every scale
        code = rng.integers(0, 0x70, (Bn, Hkv, cap, d)) if fmt == "e4m3" else rng.integers(-63, 64, (Bn, Hkv, cap, d))
        if fmt == "e4m3":
            code = code | rng.choice([0, 0x80], code.shape)
        x.view(torch.uint8).copy_(torch.from_numpy(code.astype(np.int64).astype(np.uint8)))
    q = torch.from_numpy(rng.standard_normal((Bn, G * Hkv, d)) * 0.1).to(T[dtype]).cuda()
    lists = [[np.sort(rng.choice(cap, int(rng.integers(0, cap + 1)), replace=False)).astype(np.int64) for _ in range(G * Hkv)] for _ in range(Bn)]
    for f in (heads, merged):
        check(f(c, q, lists), c, fmt, q, lists)
    check(planned(c, q, lists[:1]), c, fmt, q, [lists[0]] * Bn)


@pytest.mark.parametrize("fmt,dtype,d", FORMS)
@pytest.mark.parametrize("where", ["k", "v"])
def test_nan_rows_among_rows_of_every_size(fmt, dtype, d, where):
    """A row of NaN in a block of every size: the heads that keep one are NaN, the others as without it."""
    rng, block, cap = np.random.default_rng(85), 16, 640
    g = torch.Generator().manual_seed(85)
    of = np.repeat(rng.integers(0, 5, cap // block), block)
    c = cache(g, fmt, d, block, np.array(list(SIZES.values()))[of], torch.randn((1, 1, cap, d), generator=g))
    q = torch.randn((1, 6, d), generator=g).to(T[dtype]).cuda()
    bad = np.array([rng.choice(np.flatnonzero(of == x)) for x in range(5)])
    fine = np.setdiff1d(np.arange(cap), bad)
    lists = [[fine, np.sort(np.append(fine[of[fine] == 0], bad[4])), fine[of[fine] == 0], bad[:1], fine[of[fine] >= 2], np.arange(cap)]]
    for f in (heads, merged, planned):
        want = f(c, q, lists)
        x = B.QuantCache(c.k.clone(), c.v.clone(), c.kscale, c.vscale, block)
        getattr(x, where).view(torch.uint8)[:, :, bad] = 0x7F if fmt == "e4m3" else 0x80
        got = f(x, q, lists)
        torch.cuda.synchronize()
        assert all(torch.equal(a[:, [0, 2, 4]], b[:, [0, 2, 4]]) for a, b in zip(got, want))
        assert torch.isnan(got[0][:, [1, 3, 5]]).all()
        if where == "k":
            assert torch.isnan(got[1][:, [1, 3, 5]]).all()
        else:  # lse is of the logits alone. A sum may be held in another range without the row: where it is handed on an
            # exponential and a product, 3 u, on either side, and the roundings of the reference and the logarithm, 4 u (1 + |lse|)
            assert ((got[1] - want[1]).abs() <= 16 * U * (1 + want[1].abs())).all()
