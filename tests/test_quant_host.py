"""Refusals of the 8-bit cache's entry points: argument errors are found on the host and nothing is launched (no GPU here)."""
import ctypes

import pytest
import torch

from paper_2506_11104_amd import binding as B


def i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


def cache(**kw):
    c = B.QuantCacheView(4096, 4096, 4096, 4096, B.DAM_KV_E4M3, 64, i64(2 * 16, 16))
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(**kw):
    p = B.QuantParams(2, 2, 1024, 128, B.DAM_BF16, 10, 0, i64(2 * 10 * 128, 10 * 128, 128), i64(2 * 10 * 128, 10 * 128, 128),
                      i64(2 * 1024 * 128, 1024 * 128, 128))
    for k, v in kw.items():
        setattr(p, k, v)
    return p


WRITE_AND_READ_REFUSALS = [
    (dict(batch=0), {}, "INVALID_ARG"), (dict(hkv=0), {}, "INVALID_ARG"), (dict(kv_capacity=0), {}, "INVALID_ARG"),
    (dict(n_rows=-1), {}, "INVALID_ARG"), (dict(pos=-1), {}, "INVALID_ARG"), (dict(pos=1025), {}, "INVALID_ARG"),
    (dict(pos=1015), {}, "INVALID_ARG"),                        # ten rows from there lie behind the cache's end
    (dict(dtype=2), {}, "UNSUPPORTED"), (dict(head_dim=96), {}, "UNSUPPORTED"), (dict(head_dim=256), {}, "UNSUPPORTED"),
    (dict(kv_capacity=2**31 - 1), {}, "UNSUPPORTED"),
    (dict(k_stride=i64(2560, 1280, 130)), {}, "INVALID_ARG"), (dict(v_stride=i64(2560, 1284, 128)), {}, "INVALID_ARG"),
    (dict(kv_stride=i64(2 * 1024 * 128, 1024 * 128, 136)), {}, "INVALID_ARG"),
    (dict(k_stride=i64(-2560, 1280, 128)), {}, "INVALID_ARG"),
    ({}, dict(format=2), "UNSUPPORTED"), ({}, dict(block=8), "UNSUPPORTED"), ({}, dict(block=48), "UNSUPPORTED"),
    ({}, dict(block=0), "UNSUPPORTED"), ({}, dict(kcache=None), "INVALID_ARG"), ({}, dict(vscale=None), "INVALID_ARG"),
    ({}, dict(vcache=4104), "INVALID_ARG"), ({}, dict(scale_stride=i64(-1, 16)), "INVALID_ARG"),
]


@pytest.mark.parametrize("p,c,status", WRITE_AND_READ_REFUSALS)
def test_write_and_read_refuse(p, c, status):
    want = getattr(B, "DAM_ERR_" + status)
    L = B.lib()
    assert L.dam_kv_quantize(ctypes.byref(rows(**p)), ctypes.byref(cache(**c)), 4096, 4096, None, None, None) == want
    assert L.dam_kv_dequantize(ctypes.byref(rows(**p)), ctypes.byref(cache(**c)), None, None, 4096, 4096, None) == want


def test_what_is_written_may_not_lie_on_top_of_itself():
    L = B.lib()

    def both(p, c):
        return (L.dam_kv_quantize(ctypes.byref(p), ctypes.byref(c), 4096, 4096, None, None, None),
                L.dam_kv_dequantize(ctypes.byref(p), ctypes.byref(c), None, None, 4096, 4096, None))

    # one set of cache rows for all heads, scales of all sequences in one place: not to be written
    for p, c in ((rows(kv_stride=i64(2 * 1024 * 128, 0, 128)), cache()), (rows(kv_stride=i64(2 * 1024 * 128, 1024 * 128, 64)), cache()),
                 (rows(), cache(scale_stride=i64(0, 16)))):
        assert both(p, c)[0] == B.DAM_ERR_INVALID_ARG
    # k and v broadcast over the sequences may be read, not written
    assert both(rows(k_stride=i64(0, 1280, 128)), cache())[1] == B.DAM_ERR_INVALID_ARG
    assert both(rows(v_stride=i64(2560, 1280, 64)), cache())[1] == B.DAM_ERR_INVALID_ARG


def test_nothing_to_do_and_missing_arguments():
    L = B.lib()
    assert L.dam_kv_quantize(ctypes.byref(rows(n_rows=0)), ctypes.byref(cache()), None, None, None, None, None) == B.DAM_OK
    assert L.dam_kv_dequantize(ctypes.byref(rows(n_rows=0)), ctypes.byref(cache()), None, None, None, None, None) == B.DAM_OK
    assert L.dam_kv_quantize(ctypes.byref(rows()), ctypes.byref(cache()), None, 4096, None, None, None) == B.DAM_ERR_INVALID_ARG
    assert L.dam_kv_quantize(None, ctypes.byref(cache()), 4096, 4096, None, None, None) == B.DAM_ERR_INVALID_ARG
    assert L.dam_kv_dequantize(ctypes.byref(rows()), None, None, None, 4096, 4096, None) == B.DAM_ERR_INVALID_ARG
    assert L.dam_kv_quantize(ctypes.byref(rows()), ctypes.byref(cache()), 4100, 4096, None, None, None) == B.DAM_ERR_INVALID_ARG


def decode(**kw):
    p = B.DecodeParams()
    p.batch, p.hq, p.hkv, p.kv_capacity, p.head_dim, p.dtype, p.scale = 2, 4, 2, 1024, 128, B.DAM_BF16, 0.0
    p.q_stride, p.kv_stride, p.o_stride = i64(512, 128), i64(2 * 1024 * 128, 1024 * 128, 128), i64(512, 128)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def decode_calls(p, c, ws=4096, ws_bytes=1 << 30, member=4096, table=4096, n_flags=100, pos=50, idx=4096, most=100, q=4096):
    L = B.lib()
    p, c = ctypes.byref(p), ctypes.byref(c)
    return (L.dam_sparse_attn_decode_quantized(p, q, c, 4096, idx, most, 4096, None, ws, ws_bytes, None),
            L.dam_sparse_attn_decode_grouped_quantized(p, q, c, 4096, idx, member, most, 4096, None, ws, ws_bytes, None),
            L.dam_sparse_attn_decode_patterns_quantized(p, q, c, 4096, idx, member, table, n_flags, pos, most, 4096, None, ws,
                                                        ws_bytes, None))


@pytest.mark.parametrize("p,c,kw,status", [
    (dict(batch=0), {}, {}, "INVALID_ARG"), (dict(hq=5), {}, {}, "INVALID_ARG"), (dict(kv_capacity=0), {}, {}, "INVALID_ARG"),
    (dict(scale=-1.0), {}, {}, "INVALID_ARG"), (dict(scale=float("nan")), {}, {}, "INVALID_ARG"),
    (dict(dtype=3), {}, {}, "UNSUPPORTED"), (dict(head_dim=80), {}, {}, "UNSUPPORTED"),
    (dict(q_stride=i64(512, 132)), {}, {}, "INVALID_ARG"), (dict(kv_stride=i64(2 * 1024 * 128, 1024 * 128, 120)), {}, {}, "INVALID_ARG"),
    ({}, dict(format=-1), {}, "UNSUPPORTED"), ({}, dict(block=256), {}, "UNSUPPORTED"), ({}, dict(kscale=None), {}, "INVALID_ARG"),
    ({}, dict(kcache=4097), {}, "INVALID_ARG"), ({}, {}, dict(q=None), "INVALID_ARG"), ({}, {}, dict(idx=None), "INVALID_ARG"),
    ({}, {}, dict(most=-1), "INVALID_ARG"), ({}, {}, dict(ws=None), "WORKSPACE"), ({}, {}, dict(ws_bytes=8), "WORKSPACE"),
])
def test_decodes_refuse(p, c, kw, status):
    assert set(decode_calls(decode(**p), cache(**c), **kw)) == {getattr(B, "DAM_ERR_" + status)}


def test_grouped_decodes_refuse():
    assert decode_calls(decode(), cache(), member=None)[1:] == (B.DAM_ERR_INVALID_ARG,) * 2
    assert decode_calls(decode(hq=18, q_stride=i64(18 * 128, 128)), cache())[1:] == (B.DAM_ERR_UNSUPPORTED,) * 2
    for kw in (dict(table=None), dict(n_flags=0), dict(pos=-1), dict(pos=1024)):
        assert decode_calls(decode(), cache(), **kw)[2] == B.DAM_ERR_INVALID_ARG


def test_more_heads_than_a_launch_holds_are_refused():
    for kw in (dict(batch=1 << 22), dict(batch=(1 << 31) - 1, hq=8, hkv=8), dict(batch=1 << 20, hq=8, hkv=1),
               dict(batch=1, hq=1 << 20, hkv=1)):
        assert set(decode_calls(decode(**kw), cache(), ws_bytes=1 << 62)) == {B.DAM_ERR_UNSUPPORTED}, kw


def test_one_workspace_for_a_batch_that_shrinks():
    L = B.lib()
    for hq, hkv, d, dtype in ((32, 8, 128, B.DAM_BF16), (16, 16, 64, B.DAM_F32), (64, 8, 128, B.DAM_BF16), (3, 1, 64, B.DAM_BF16)):
        p = decode(hq=hq, hkv=hkv, head_dim=d, dtype=dtype, kv_capacity=70000)
        for query in (L.dam_sparse_attn_decode_quantized_workspace, L.dam_sparse_attn_decode_grouped_quantized_workspace):
            for n in (40, 700, 6000, 70000):
                sizes = []
                for p.batch in (*range(1, 70), 128, 500, 1023, 1024, 1025, 3000):
                    sizes.append(query(ctypes.byref(p), n))
                assert sizes == sorted(sizes) and sizes[0] > 0, (hq, hkv, n, sizes)
            p.batch = 4
            sizes = [query(ctypes.byref(p), n) for n in (0, 1, 40, 200, 300, 700, 3000, 70000)]
            assert sizes == sorted(sizes)
        p.hq = 5 * hkv + 1
        if hkv > 1:
            assert query(ctypes.byref(p), 100) == 0


def test_tensors_that_do_not_fit_together_are_refused():
    """Shapes, types and places of the tensors, found before anything is launched."""
    c = B.quant_cache(2, 2, 100, 128, block=32, device="cpu")
    k = torch.zeros(2, 2, 5, 128, dtype=torch.bfloat16)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(AssertionError, match="current device"):
        B.dam_kv_quantize(c, k, k)                                           # host memory
    for a, b in ((k[:1], k[:1]), (k[..., :64], k[..., :64]), (k, k[:, :, :4]), (k[:, :1], k[:, :1])):
        with pytest.raises(AssertionError, match="fit together"):
            B.dam_kv_quantize(c, a, b)
    with pytest.raises(AssertionError, match="fit together"):
        B.dam_kv_quantize(c, k, k, start=i32(1))
    with pytest.raises(AssertionError, match="fit together"):
        B.dam_kv_quantize(c, k, k, count=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(B.DamError):
        B.dam_kv_quantize(c, k.half(), k.half())
    with pytest.raises(B.DamError):
        B.dam_kv_dequantize(c, k, k.float())
    for other in (B.QuantCache(c.k, c.v.view(torch.int8), c.kscale, c.vscale, 32), B.QuantCache(c.k, c.v, c.kscale.view(torch.int8), c.vscale, 32),
                  B.QuantCache(c.k.view(torch.uint8), c.v.view(torch.uint8), c.kscale, c.vscale, 32)):
        with pytest.raises(B.DamError):
            B.dam_kv_quantize(other, k, k)
    for other in (B.QuantCache(c.k, c.v, c.kscale, c.vscale, 16), B.QuantCache(c.k, c.v, c.kscale[:, :, ::2], c.vscale[:, :, ::2], 64),
                  B.QuantCache(c.k, c.v, c.kscale, c.vscale[:1], 32), B.QuantCache(c.k, c.v[:, :, :99], c.kscale, c.vscale, 32)):
        with pytest.raises(AssertionError, match="fit together"):
            B.dam_kv_quantize(other, k, k)
    q = torch.zeros(2, 4, 128, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    with pytest.raises(AssertionError, match="current device"):
        B.dam_sparse_attn_decode_quantized(q, c, i32(9), i32(4), 4, ws=ws)
    for kw in (dict(kept_ptr=i32(8)), dict(kept_idx=torch.zeros(4, dtype=torch.int64)), dict(lse=torch.zeros(2, 3)),
               dict(q=q[:1]), dict(q=q[..., :64]), dict(out=torch.zeros(2, 3, 128, dtype=torch.bfloat16))):
        with pytest.raises(AssertionError, match="fit together"):
            B.dam_sparse_attn_decode_quantized(**{**dict(q=q, cache=c, kept_ptr=i32(9), kept_idx=i32(4), max_kept=4, ws=ws), **kw})
    with pytest.raises(AssertionError, match="member"):
        B.dam_sparse_attn_decode_grouped_quantized(q, c, i32(5), i32(4), None, 4, ws=ws)
    with pytest.raises(B.DamError):
        B.dam_sparse_attn_decode_quantized(q, c, i32(9), i32(4), 4, out=q.float(), ws=ws)
    with pytest.raises(B.DamError):
        B.dam_sparse_attn_decode_quantized(q.half(), c, i32(9), i32(4), 4, ws=ws)


def test_a_tensor_without_memory_is_a_python_error():
    nat = B.native()
    c = B.quant_cache(1, 2, 128, 128, device="cpu")
    ints = torch.zeros(8, dtype=torch.int32)
    for call in (lambda t: nat.kv_rows(c.k, c.v, c.kscale, c.vscale, 64, t, t, 0, None, None, True),
                 lambda t: nat.decode_quantized(c.k, c.v, c.kscale, c.vscale, 64, t[0], ints, ints, None, 4, t[0], None, 0.0, True, None),
                 lambda t: nat.decode_patterns_quantized(c.k, c.v, c.kscale, c.vscale, 64, t[0], ints, ints, None,
                                                         torch.zeros(2, 4, dtype=torch.uint8), 3, 4, t[0], None, 0.0, None)):
        with pytest.raises((RuntimeError, AssertionError)):
            torch.vmap(lambda t: B._check("the call", call(t)))(torch.zeros(3, 1, 2, 4, 128, dtype=torch.bfloat16))
