"""The decodes over a cache of 8-bit codes on the GPU against the oracle in 64 bits, in every form.

Tolerances. With n kept keys, z the logits, Z = max_j scale sum_d |q_d k_jd|, A = sum_j p_j |v_j| and u = 2^-24:
  - a logit is a sum of d products in fp32 and two multiplications: |dz| <= (d + 4) u Z, and each weight exp(z - m) is off by
    that of z and of m, by the rounding of its own exponent (|z - m| <= 2 Z: 4 u Z) and by 2 u of the exponential itself:
    dw <= (2 d + 16) u Z + 4 u relative;
  - weights and products are summed in fp32 in whatever order: n u of the sums, each, and a few more for the merges: (n + 64) u;
  - 32 bits end at 2^-126: a weight below is taken as 0, off by less than that, and so is its product with a value's scale,
    which a code of at most 448 multiplies: n 2^-126 (max |v| + 448) of the sums, whose largest weight is 1;
  - where the products run on the matrix cores (bf16 queries) the weights go in as two bf16 terms, off by at most 2^-16.
  So |dO| <= A (2 dw + 2 (n + 64) u + 2^-16 [bf16]) + n 2^-126 (max |v| + 448) + 2^-8 |O| [bf16: half a step of the output],
     |dlse| <= (d + 4) u Z + dw + (n + 64) u + 2^-22 (1 + |lse|)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import quant as oq
from paper_2506_11104_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
T = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda() if len(a) else torch.zeros(1, dtype=torch.int32, device="cuda")


def u8(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.uint8)).cuda() if len(a) else torch.zeros(1, dtype=torch.uint8, device="cuda")


def make(seed, fmt, dtype, Bn, Hq, Hkv, d, cap, block, spread=1.0):
    """A cache whose blocks have scales of their own, and queries."""
    g = torch.Generator().manual_seed(seed)
    c = B.quant_cache(Bn, Hkv, cap, d, DTYPE[fmt], block)
    k, v = ((torch.randn((Bn, Hkv, cap, d), generator=g) * torch.exp(spread * (2 * torch.rand((Bn, Hkv, cap, 1), generator=g) - 1))).cuda()
            for _ in range(2))
    B.dam_kv_quantize(c, k, v)
    q = (1.5 * torch.randn((Bn, Hq, d), generator=g)).to(T[dtype]).cuda()
    return c, q


def cache_values(c, fmt):
    torch.cuda.synchronize()
    return [oq.values(x.view(torch.uint8).cpu().numpy(), s.cpu().numpy(), c.block, fmt) for x, s in ((c.k, c.kscale), (c.v, c.vscale))]


def check(got, c, fmt, q, lists, scale=None):
    """lists[b][h]: the keys that query head h of sequence b keeps."""
    out, lse = (x.double().cpu().numpy() for x in got)
    K, V = cache_values(c, fmt)
    qh = q.double().cpu().numpy()
    Bn, Hq, d = qh.shape
    G = Hq // K.shape[1]
    bf16 = q.dtype == torch.bfloat16
    for b in range(Bn):
        for h in range(Hq):
            keys = lists[b][h]
            O, L, A, Z = oq.attend(qh[b, h], K[b, h // G], V[b, h // G], keys, scale)
            n, where = len(keys), f"sequence {b} head {h}, {len(keys)} keys"
            if n == 0:
                assert (out[b, h] == 0).all() and lse[b, h] == -np.inf, where
                continue
            assert np.array_equal(np.isnan(out[b, h]), np.isnan(O)) and np.isnan(lse[b, h]) == np.isnan(L), where
            if np.isnan(L):
                continue
            fine = ~np.isnan(O)
            dw = (2 * d + 16) * U * Z + 4 * U
            tol = A * (2 * dw + 2 * (n + 64) * U + (2.0 ** -16 if bf16 else 0)) + (2.0 ** -8 * np.abs(O) if bf16 else U * np.abs(O))
            tol = tol + n * 2.0 ** -126 * (np.nanmax(np.abs(V[b, h // G][keys])) + 448)
            err = np.abs(out[b, h] - O)
            assert (err[fine] <= tol[fine]).all(), f"{where}: {np.nanmax(err / tol):.2f} of the bound"
            assert abs(lse[b, h] - L) <= (d + 4) * U * Z + dw + (n + 64) * U + 2.0 ** -22 * (1 + abs(L)), where


def heads(c, q, lists, shared=False, **kw):
    flat = [lists[0][h] for h in range(q.shape[1])] if shared else [x for b in lists for x in b]
    ptr = np.concatenate([[0], np.cumsum([len(x) for x in flat])])
    return B.dam_sparse_attn_decode_quantized(q, c, i32(ptr), i32(np.concatenate(flat)), max(len(x) for x in flat), want_lse=True,
                                              shared_lists=shared, **kw)


def merged(c, q, lists, shared=False, shuffle=None, **kw):
    flat = [lists[0][h] for h in range(q.shape[1])] if shared else [x for b in lists for x in b]
    ptr, idx, mem = oracle.group_lists(flat, q.shape[1] // c.k.shape[1])
    if shuffle is not None:  # entries of a list may come in any order
        for a, b in zip(ptr[:-1], ptr[1:]):
            o = shuffle.permutation(b - a)
            idx[a:b], mem[a:b] = idx[a:b][o], mem[a:b][o]
    return B.dam_sparse_attn_decode_grouped_quantized(q, c, i32(ptr), i32(idx), u8(mem), int(np.diff(ptr).max()), want_lse=True,
                                                      shared_lists=shared, **kw)


def pick(rng, cap, lens):
    return [np.sort(rng.choice(cap, int(n), replace=False)).astype(np.int64) for n in lens]


@pytest.mark.parametrize("block", [16, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_small_and_ragged_lists(fmt, dtype, d, block):
    rng = np.random.default_rng(41)
    Bn, Hq, Hkv, cap = 3, 4, 2, 700
    c, q = make(41, fmt, dtype, Bn, Hq, Hkv, d, cap, block)
    lens = rng.integers(0, 300, Bn * Hq)
    lens[:6] = 0, 1, 3, 700, 33, 32
    lens[8:10] = 0
    flat = pick(rng, cap, lens)
    lists = [flat[b * Hq:(b + 1) * Hq] for b in range(Bn)]
    check(heads(c, q, lists), c, fmt, q, lists)
    check(merged(c, q, lists), c, fmt, q, lists)


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "bf16", 128), ("int8", "f32", 128), ("e4m3", "bf16", 64)])
def test_groups_of_every_size(fmt, dtype, d, G):
    rng = np.random.default_rng(42 + G)
    Bn, Hkv, cap = 2, 2, 400
    c, q = make(42, fmt, dtype, Bn, G * Hkv, Hkv, d, cap, 32)
    common = rng.choice(cap, 60, replace=False)
    lists = [[np.unique(np.concatenate([common[:rng.integers(0, 60)], rng.choice(cap, rng.integers(0, 80), replace=False)]))
              for _ in range(G * Hkv)] for _ in range(Bn)]
    check(merged(c, q, lists, shuffle=rng), c, fmt, q, lists)
    check(merged(c, q, lists[:1] * Bn, shared=True), c, fmt, q, lists[:1] * Bn)
    check(heads(c, q, lists[:1] * Bn, shared=True), c, fmt, q, lists[:1] * Bn)


@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "bf16", 128), ("e4m3", "f32", 64), ("int8", "bf16", 64)])
@pytest.mark.parametrize("Bn,Hq,Hkv,lens", [
    (1, 4, 1, (9000, 8191, 1, 4097)), (1, 8, 8, (33, 9000, 0, 512, 5000, 1, 31, 257)), (1, 8, 1, (3000,) * 8),
    (2, 4, 2, (1500, 40, 0, 6000, 2, 700, 900, 5)), (40, 8, 4, tuple(range(0, 320 * 3, 3)))])
def test_long_lists_use_many_splits(fmt, dtype, d, Bn, Hq, Hkv, lens):
    rng = np.random.default_rng(43)
    cap = 9000 if max(lens) > 1000 else 1000
    c, q = make(43, fmt, dtype, Bn, Hq, Hkv, d, cap, 64)
    flat = pick(rng, cap, lens)
    lists = [flat[b * Hq:(b + 1) * Hq] for b in range(Bn)]
    check(heads(c, q, lists), c, fmt, q, lists)
    check(merged(c, q, lists), c, fmt, q, lists)


@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "bf16", 128), ("int8", "f32", 64), ("e4m3", "bf16", 64)])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_plans_at_every_kind_of_position(fmt, dtype, d, G):
    """Positions in front of most patterns, in the middle, beyond the flags' length; rows that do not exist yet hold NaN."""
    rng = np.random.default_rng(44 + G)
    Hkv, Bn, P, cap = 2, 2, 500, 900
    Hq = G * Hkv
    dflag = (rng.random((Hq, P)) < 0.04).astype(np.uint8)
    vflag = (rng.random((Hq, P)) < 0.04).astype(np.uint8)
    dflag[:, :40] = 1
    vflag[:, :3] = 1
    dflag[0], vflag[0] = 0, 0
    ptr, val, mem, table = oracle.pattern_plan(dflag, vflag, G)
    plan = B.Mask(H=Hq, L=0, S=P, tile_m=128, tile_n=128, kept_ptr=i32(ptr), kept_idx=i32(val), kept_member=u8(mem),
                  plan_table=u8(table))
    most = int(np.diff(ptr).max())
    c, q = make(44, fmt, dtype, Bn, Hq, Hkv, d, cap, 32)
    ws = B.decode_quantized_workspace(q, c, most, True, True)
    for pos in (0, 1, 31, 250, 499, 700, 899):
        keep = [[np.array([j for j in range(pos + 1) if (pos - j < P and dflag[h, pos - j]) or (j < P and vflag[h, j])], np.int64)
                 for h in range(Hq)]] * Bn
        later = B.QuantCache(c.k.clone(), c.v.clone(), c.kscale.clone(), c.vscale.clone(), c.block)
        for x in (later.k, later.v):
            x.view(torch.uint8)[:, :, pos + 1:] = 0x7F if fmt == "e4m3" else 0x80
        got = B.dam_sparse_attn_decode_patterns_quantized(q, later, plan, pos, most, want_lse=True, ws=ws)
        check(got, later, fmt, q, keep)


@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "bf16", 128), ("int8", "f32", 64), ("e4m3", "f32", 128),
                                         ("int8", "bf16", 64)])
@pytest.mark.parametrize("where", ["k", "v"])
def test_nan_rows_reach_the_heads_that_keep_them_alone(fmt, dtype, d, where):
    rng = np.random.default_rng(45)
    Bn, Hq, Hkv, cap = 2, 8, 2, 600
    g = torch.Generator().manual_seed(45)
    c = B.quant_cache(Bn, Hkv, cap, d, DTYPE[fmt], 16)
    k, v = (torch.randn((Bn, Hkv, cap, d), generator=g).cuda() for _ in range(2))
    bad = rng.choice(cap, 12, replace=False)
    for i, r in enumerate(bad):
        (k if where == "k" else v)[i % 2, i % 3 % 2, r, i % d] = (float("nan"), float("inf"), float("-inf"))[i % 3]
    B.dam_kv_quantize(c, k, v)
    q = torch.randn((Bn, Hq, d), generator=g).to(T[dtype]).cuda()
    lists = [pick(rng, cap, rng.integers(1, 90, Hq)) for _ in range(Bn)]
    lists[0][0] = np.sort(bad[:5])                       # nothing but NaN rows, in one of the two KV heads
    lists[1][1] = np.setdiff1d(np.arange(cap), bad)      # everything else
    lists[1][6] = bad[:1]
    for f in (heads, merged):
        got = f(c, q, lists)
        check(got, c, fmt, q, lists)
    n = torch.isnan(got[0].float()).any(-1)
    assert n.any() and not n.all()


@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "bf16", 128), ("e4m3", "f32", 64)])
def test_logits_that_stand_far_apart_and_far_from_zero(fmt, dtype, d):
    """Scaled logits of a few hundred of either sign, a sink whose values are zero, values of very different scales."""
    rng = np.random.default_rng(46)
    Bn, Hq, Hkv, cap, block = 1, 4, 1, 1200, 32
    g = torch.Generator().manual_seed(46)
    c = B.quant_cache(Bn, Hkv, cap, d, DTYPE[fmt], block)
    k, v = (torch.randn((Bn, Hkv, cap, d), generator=g).cuda() for _ in range(2))
    q = torch.randn((Bn, Hq, d), generator=g).to(T[dtype]).cuda()
    k[0, 0, 300:700] *= 30
    k[0, 0, 5] = 30 * q[0, 1].float()
    v[0, 0, :32] = 0                                      # (a whole block: its scale is 0)
    v[0, 0, 400:800] *= 1e4
    v[0, 0, 800:1000] *= 1e-4
    B.dam_kv_quantize(c, k, v)
    lists = [pick(rng, cap, (1200, 500, 900, 40))]
    lists[0][1] = np.union1d(lists[0][1], [5])
    for f in (heads, merged):
        check(f(c, q, lists), c, fmt, q, lists)
        check(f(c, q, lists, scale=-0.0 + 0.01), c, fmt, q, lists, scale=np.float32(0.01))


@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "f32", 64)])
def test_layouts_other_than_the_dense_one(fmt, dtype, d):
    """Position-major caches with K and V rows side by side, scales, queries and outputs as slices: the same bits."""
    rng = np.random.default_rng(47)
    Bn, Hq, Hkv, cap, block = 3, 8, 2, 500, 16
    c, q = make(47, fmt, dtype, Bn, Hq, Hkv, d, cap, block)
    both = torch.zeros((Bn, cap, Hkv, 2, d), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((Bn, Hkv, 2, 40), dtype=torch.uint8, device="cuda")
    c2 = B.QuantCache(*(both[:, :, :, i].transpose(1, 2).view(DTYPE[fmt]) for i in (0, 1)), scales[:, :, 0], scales[:, :, 1], block)
    for a, b in ((c.k, c2.k), (c.v, c2.v)):
        b.view(torch.uint8).copy_(a.view(torch.uint8))
    for a, b in ((c.kscale, c2.kscale), (c.vscale, c2.vscale)):
        b[..., :a.shape[2]] = a
    wide = torch.zeros((Bn, 2, Hq, d + 8), dtype=q.dtype, device="cuda")
    q2, out2 = wide[:, 0, :, :d], torch.zeros((Hq, Bn, 3 * d), dtype=q.dtype, device="cuda").transpose(0, 1)[..., d:2 * d]
    q2.copy_(q)
    lists = [pick(rng, cap, rng.integers(0, 400, Hq)) for _ in range(Bn)]
    for f in (heads, merged):
        want, want_lse = f(c, q, lists)
        got, lse = f(c2, q2, lists, out=out2)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(lse, want_lse)


def test_indexes_outside_the_cache_read_its_nearest_row():
    c, q = make(48, "e4m3", "bf16", 1, 4, 1, 128, 100, 16)
    ptr, wild, tame = i32([0, 4]), i32([-5, 3, 99, 1 << 30]), i32([0, 3, 99, 99])
    mem = u8([15, 15, 15, 15])
    a = B.dam_sparse_attn_decode_grouped_quantized(q, c, ptr, wild, mem, 4)
    b = B.dam_sparse_attn_decode_grouped_quantized(q, c, ptr, tame, mem, 4)
    per = i32([0, 4, 4, 4, 4])
    e = B.dam_sparse_attn_decode_quantized(q, c, per, wild, 4)
    f = B.dam_sparse_attn_decode_quantized(q, c, per, tame, 4)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(e, f)


def test_a_cache_of_more_than_four_gigabytes_a_head():
    """Keys on either side of 2^32 bytes from the head's first row."""
    cap, d = (1 << 25) + 200, 128
    c = B.quant_cache(1, 1, cap, d, torch.int8, 128)
    g = torch.Generator().manual_seed(49)
    k, v = (torch.randn((1, 1, 300, d), generator=g).cuda() for _ in range(2))
    lo = (1 << 25) - 100
    B.dam_kv_quantize(c, k, v, pos=lo - lo % 128)
    small = B.quant_cache(1, 1, 384, d, torch.int8, 128)
    B.dam_kv_quantize(small, k, v)
    q = torch.randn((1, 4, d), generator=g).to(torch.bfloat16).cuda()
    keys = np.arange(0, 300, 2)
    ptr, mem = i32([0, len(keys)]), u8([15] * len(keys))
    a = B.dam_sparse_attn_decode_grouped_quantized(q, c, ptr, i32(keys + lo - lo % 128), mem, len(keys))
    b = B.dam_sparse_attn_decode_grouped_quantized(q, small, ptr, i32(keys), mem, len(keys))
    per = i32([0] + [len(keys)] * 4)
    e = B.dam_sparse_attn_decode_quantized(q, c, per, i32(keys + lo - lo % 128), len(keys))
    f = B.dam_sparse_attn_decode_quantized(q, small, per, i32(keys), len(keys))
    torch.cuda.synchronize()
    assert torch.equal(e, f)
    assert torch.equal(a, b)
    # from a plan: 150 diagonals and twenty columns, from a position behind the border
    pos, base = lo - lo % 128 + 299, lo - lo % 128
    val = np.concatenate([-1 - np.arange(149, -1, -1), np.arange(20) + base])
    table = np.zeros((1, 300), np.uint8)
    table[0, :150] = 15

    def decode(cache, at, shift):
        v = np.where(val < 0, val, val - shift)
        plan = B.Mask(H=4, L=0, S=300, tile_m=128, tile_n=128, kept_ptr=i32([0, len(v)]), kept_idx=i32(v),
                      kept_member=u8([15] * len(v)), plan_table=u8(table))
        return B.dam_sparse_attn_decode_patterns_quantized(q, cache, plan, at, len(v))

    x, y = decode(c, pos, 0), decode(small, 299, base)
    torch.cuda.synchronize()
    assert torch.equal(x, y)


@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "bf16", 64), ("e4m3", "f32", 64)])
def test_more_blocks_than_waves_have_and_the_same_bits_twice(fmt, dtype, d):
    """Enough long lists for workgroups of eight waves, two or more of them to a list; the second call, on another stream and
    with another workspace, gives the same bits."""
    rng = np.random.default_rng(52)
    Bn, Hq, Hkv, cap = 20, 4, 2, 8000
    c, q = make(52, fmt, dtype, Bn, Hq, Hkv, d, cap, 128)
    common = [rng.choice(cap, 6800, replace=False) for _ in range(Hkv)]
    lists = [[np.sort(common[h // 2][:6800 - 300 * (h % 2)]) for h in range(Hq)] for _ in range(Bn)]
    for f in (heads, merged):
        got = f(c, q, lists, shared=True)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            again = f(c, q, lists, shared=True)
        torch.cuda.synchronize()
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
        pick3 = [0, 7, 19]
        check([x[pick3] for x in got], B.QuantCache(c.k[pick3], c.v[pick3], c.kscale[pick3], c.vscale[pick3], 128) if fmt == "int8" else
              B.QuantCache(*(x.view(torch.uint8)[pick3].view(DTYPE[fmt]) for x in (c.k, c.v)), c.kscale[pick3], c.vscale[pick3], 128),
              fmt, q[pick3], [lists[i] for i in pick3])


@pytest.mark.parametrize("seed", range(24))
def test_random_small_configurations(seed):
    """Sizes, layouts of heads, blocks, list lengths and positions drawn; all three forms on the same cache."""
    rng = np.random.default_rng(1000 + seed)
    fmt, dtype = ("e4m3", "int8")[rng.integers(2)], ("bf16", "f32")[rng.integers(2)]
    d, block, G, Hkv, Bn = int(rng.choice([64, 128])), int(rng.choice([16, 32, 64, 128])), int(rng.integers(1, 9)), int(rng.integers(1, 4)), int(rng.integers(1, 4))
    cap = int(rng.integers(1, 700))
    Hq = G * Hkv
    c, q = make(seed, fmt, dtype, Bn, Hq, Hkv, d, cap, block, spread=3.0)
    lists = [pick(rng, cap, np.minimum(cap, rng.integers(0, 1 + cap // int(rng.integers(1, 5)), Hq))) for _ in range(Bn)]
    scale = None if seed % 3 else 0.25
    kw = {} if scale is None else {"scale": scale}
    check(heads(c, q, lists, **kw), c, fmt, q, lists, scale)
    check(merged(c, q, lists, shuffle=rng if seed % 2 else None, **kw), c, fmt, q, lists, scale)
    P = int(rng.integers(1, cap + 50))
    dflag, vflag = ((rng.random((Hq, P)) < rng.random() * 0.2).astype(np.uint8) for _ in range(2))
    ptr, val, mem, table = oracle.pattern_plan(dflag, vflag, G)
    plan = B.Mask(H=Hq, L=0, S=P, tile_m=128, tile_n=128, kept_ptr=i32(ptr), kept_idx=i32(val), kept_member=u8(mem), plan_table=u8(table))
    pos = int(rng.integers(0, cap))
    keep = [[np.array([j for j in range(pos + 1) if (pos - j < P and dflag[h, pos - j]) or (j < P and vflag[h, j])], np.int64)
             for h in range(Hq)]] * Bn
    got = B.dam_sparse_attn_decode_patterns_quantized(q, c, plan, pos, int(np.diff(ptr).max()), want_lse=True, **kw)
    check(got, c, fmt, q, keep, scale)


def test_outputs_that_lie_off_alignment():
    for dtype, d, G in (("bf16", 128, 4), ("f32", 64, 2), ("bf16", 64, 1)):
        rng = np.random.default_rng(53)
        c, q = make(53, "e4m3", dtype, 2, 2 * G, 2, d, 300, 16)
        lists = [pick(rng, 300, rng.integers(0, 200, 2 * G)) for _ in range(2)]
        for f in (heads, merged):
            want, want_lse = f(c, q, lists)
            wide = torch.full((2, 2 * G, d + 5), 7.0, dtype=q.dtype, device="cuda")
            got, lse = f(c, q, lists, out=wide[..., 1:d + 1])
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(lse, want_lse)
            assert (wide[..., 0] == 7).all() and (wide[..., d + 1:] == 7).all()


def test_a_decode_loop_from_a_graph():
    """Token by token: write the new row, decode from the plan and from the lists of the position, replayed from a graph with
    new inputs each time; every replay equals the eager calls, two graphs share a workspace, and the last step is held to
    the oracle."""
    rng = np.random.default_rng(50)
    Bn, Hq, Hkv, d, cap, block, G = 2, 8, 2, 128, 1500, 64, 4
    dflag = (rng.random((Hq, cap)) < 0.01).astype(np.uint8)
    vflag = (rng.random((Hq, cap)) < 0.01).astype(np.uint8)
    dflag[:, :200] = 1
    c, q = make(50, "e4m3", "bf16", Bn, Hq, Hkv, d, cap, block)
    ptr, val, mem, table = oracle.pattern_plan(dflag, vflag, G)
    plan = B.Mask(H=Hq, L=0, S=cap, tile_m=128, tile_n=128, kept_ptr=i32(ptr), kept_idx=i32(val), kept_member=u8(mem),
                  plan_table=u8(table))
    most, pos = int(np.diff(ptr).max()), 1400
    g = torch.Generator().manual_seed(51)
    k, v = (torch.randn((Bn, Hkv, 1, d), generator=g).cuda() for _ in range(2))
    ws = B.decode_quantized_workspace(q, c, most, True, True)
    rows_kept = [[np.array([j for j in range(pos + 1) if dflag[h, pos - j] or vflag[h, j]], np.int64) for h in range(Hq)]]
    lp, li, lm = oracle.group_lists(rows_kept[0], G)
    lp, li, lm = i32(lp), i32(li), u8(lm)
    out = [torch.empty_like(q) for _ in range(2)]
    lse = [torch.empty((Bn, Hq), device="cuda") for _ in range(2)]

    def write_and_plan():
        B.dam_kv_quantize(c, k, v, pos=pos)
        B.dam_sparse_attn_decode_patterns_quantized(q, c, plan, pos, most, out=out[0], lse=lse[0], ws=ws)

    def lists():
        B.dam_sparse_attn_decode_grouped_quantized(q, c, lp, li, lm, most, out=out[1], lse=lse[1], ws=ws, shared_lists=True)

    write_and_plan()
    lists()
    torch.cuda.synchronize()
    graphs = []
    for f in (write_and_plan, lists):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f()
        graphs.append(graph)
    for rep in range(4):
        q.copy_(torch.randn((Bn, Hq, d), generator=g).to(torch.bfloat16))
        k.copy_(torch.randn((Bn, Hkv, 1, d), generator=g) * (1 + rep))
        for x in graphs:
            x.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out + lse]
        write_and_plan()
        lists()
        torch.cuda.synchronize()
        for a, b in zip(got, out + lse):
            assert torch.equal(a, b), rep
    for o, l in zip(out, lse):
        check((o, l), c, "e4m3", q, rows_kept * Bn)


@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "f32", 128), ("e4m3", "f32", 64)])
def test_keys_listed_more_than_once_count_as_often(fmt, dtype, d):
    rng = np.random.default_rng(54)
    Bn, Hq, Hkv, cap, G = 2, 4, 2, 200, 2
    c, q = make(54, fmt, dtype, Bn, Hq, Hkv, d, cap, 32)
    lists = [[rng.integers(0, cap, n).astype(np.int64) for n in row] for row in ((2, 300, 65, 0), (1, 33, 500, 32))]
    lists[0][0][:] = 7
    check(heads(c, q, lists), c, fmt, q, lists)
    idx, mem, ptr = [], [], [0]
    for b in range(Bn):
        for h in range(Hkv):
            for x in range(G):
                idx.append(lists[b][h * G + x]), mem.append(np.full(len(idx[-1]), 1 << x))
            ptr.append(sum(len(x) for x in idx))
    got = B.dam_sparse_attn_decode_grouped_quantized(q, c, i32(ptr), i32(np.concatenate(idx)), u8(np.concatenate(mem)),
                                                     int(np.diff(ptr).max()), want_lse=True)
    check(got, c, fmt, q, lists)


@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "f32", 64)])
def test_a_cache_of_one_row_and_blocks_larger_than_the_cache(fmt, dtype, d):
    for cap, block in ((1, 16), (1, 128), (17, 128), (33, 32)):
        c, q = make(55, fmt, dtype, 1, 3, 1, d, cap, block)
        lists = [[np.arange(cap), np.arange(0), np.arange(cap - 1, cap)]]
        for f in (heads, merged):
            check(f(c, q, lists), c, fmt, q, lists)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("fmt,dtype,d", [("e4m3", "bf16", 128), ("int8", "f32", 128), ("e4m3", "f32", 64), ("int8", "bf16", 64)])
def test_a_query_that_is_not_finite_stays_alone(fmt, dtype, d, value):
    rng = np.random.default_rng(56)
    Bn, Hq, Hkv, cap = 1, 6, 2, 900
    c, q = make(56, fmt, dtype, Bn, Hq, Hkv, d, cap, 64)
    lists = [pick(rng, cap, [500, 40, 300, 900, 31, 200])]
    bad = q.clone()
    bad[0, 1, 5] = value
    rest = [0, 2, 3, 4, 5]
    for f in (heads, merged):
        want, want_lse = f(c, q, lists)
        got, lse = f(c, bad, lists)
        torch.cuda.synchronize()
        assert torch.equal(got[:, rest], want[:, rest]) and torch.equal(lse[:, rest], want_lse[:, rest])
        assert torch.isnan(got[0, 1]).all()


def test_two_calls_at_once():
    """On two streams, each with a workspace of its own, many times over: the results of the calls alone."""
    rng = np.random.default_rng(57)
    cap = 6000
    c, _ = make(57, "e4m3", "bf16", 2, 8, 2, 128, cap, 64)
    qs = [torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(s)).to(torch.bfloat16).cuda() for s in (58, 59)]
    lists = [[pick(rng, cap, rng.integers(1000, 3000, 8)) for _ in range(2)] for _ in qs]
    calls = []
    for q, ls in zip(qs, lists):
        ptr, idx, mem = oracle.group_lists([x for b in ls for x in b], 4)
        most = int(np.diff(ptr).max())
        calls.append((q, c, i32(ptr), i32(idx), u8(mem), most))
    ws = [B.decode_quantized_workspace(q, c, a[5], True) for q, a in zip(qs, calls)]
    outs = [torch.empty((20, *q.shape), dtype=q.dtype, device="cuda") for q in qs]
    want = [B.dam_sparse_attn_decode_grouped_quantized(*a, ws=w).clone() for a, w in zip(calls, ws)]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    for i in range(20):
        for s, a, w, o in zip(streams, calls, ws, outs):
            with torch.cuda.stream(s):
                B.dam_sparse_attn_decode_grouped_quantized(*a, ws=w, out=o[i])
    torch.cuda.synchronize()
    for o, x in zip(outs, want):
        assert all(torch.equal(y, x) for y in o)


@pytest.mark.parametrize("fill", [0, 1, 0x7F, 0xFF, None])
def test_workspaces_that_hold_anything(fill):
    rng = np.random.default_rng(60)
    cap = 5000
    c, q = make(60, "e4m3", "bf16", 1, 4, 2, 128, cap, 64)
    lists = [pick(rng, cap, [3000, 5000, 0, 4000])]
    most = 2 * cap
    want = [f(c, q, lists) for f in (heads, merged)]
    for grouped, f, x in zip((False, True), (heads, merged), want):
        ws = B.decode_quantized_workspace(q, c, most, grouped)
        for rep in range(3):
            if fill is None:
                ws.copy_(torch.from_numpy(rng.integers(0, 256, ws.numel()).astype(np.uint8)))
            else:
                ws.fill_(fill)
            for _ in range(2):  # and as the call left it
                got = f(c, q, lists, ws=ws)
                torch.cuda.synchronize()
                assert torch.equal(got[0], x[0]) and torch.equal(got[1], x[1])
    check(want[0], c, "e4m3", q, lists)
    check(want[1], c, "e4m3", q, lists)
