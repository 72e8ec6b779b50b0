"""Lists whose entries end where their 32-bit offsets do: at 2^31 - 1, in the middle of a block of 32 entries. The same entries
at the front of an array give the same bits."""
import pytest
import torch

from paper_2506_11104_amd import binding as B

pytestmark = pytest.mark.gpu
END, N, CAP, D, G = (1 << 31) - 1, 70, 200, 128, 4


@pytest.fixture(scope="module")
def entries():
    """(indexes, member bits of the last N entries, of the last one alone): the entries in front of the last N are row 0, of no head."""
    idx = torch.zeros(END, dtype=torch.int32, device="cuda")
    mem, one = (torch.zeros(END, dtype=torch.uint8, device="cuda") for _ in range(2))
    idx[-N:] = torch.arange(3, 3 + 2 * N, 2, dtype=torch.int32)
    mem[-N:] = torch.arange(N).remainder(15).add(1).to(torch.uint8)
    one[-1] = 15
    yield idx, mem, one
    del idx, mem, one
    torch.cuda.empty_cache()


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def decodes(form):
    """f(ptr, idx, mem, longest) -> (out, lse)."""
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((1, 1, CAP, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn((1, G, D), generator=g).to(torch.bfloat16).cuda()
    c = B.quant_cache(1, 1, CAP, D, torch.int8, 64)
    B.dam_kv_quantize(c, k, v)
    table = torch.zeros((1, 8), dtype=torch.uint8, device="cuda")

    def f(ptr, idx, mem, longest):
        plan = B.Mask(H=G, L=0, S=8, tile_m=128, tile_n=128, kept_ptr=ptr, kept_idx=idx, kept_member=mem, plan_table=table)
        if form == "merged":
            return B.dam_sparse_attn_decode_grouped(q, k, v, ptr, idx, mem, longest, want_lse=True, shared_lists=True)
        if form == "plan":
            return B.dam_sparse_attn_decode_patterns(q, k, v, plan, CAP - 1, longest, want_lse=True)
        if form == "merged, 8 bits":
            return B.dam_sparse_attn_decode_grouped_quantized(q, c, ptr, idx, mem, longest, want_lse=True, shared_lists=True)
        return B.dam_sparse_attn_decode_patterns_quantized(q, c, plan, CAP - 1, longest, want_lse=True)

    return f


FORMS = ["merged", "plan", "merged, 8 bits", "plan, 8 bits"]


@pytest.mark.parametrize("form", FORMS)
def test_a_list_that_ends_with_the_offsets(entries, form):
    idx, mem, _ = entries
    f = decodes(form)
    for n in (N, 33, 1):
        want = f(i32(0, n), idx[-n:].clone(), mem[-n:].clone(), N)
        got = f(i32(END - n, END), idx, mem, N)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), n


@pytest.mark.parametrize("form", FORMS)
def test_a_list_as_long_as_offsets_allow(entries, form):
    """Of its 2^31 - 1 entries the last one alone belongs to heads: its row of V comes out as it is."""
    idx, _, one = entries
    f = decodes(form)
    want = f(i32(0, 1), idx[-1:].clone(), one[-1:].clone(), END)
    got = f(i32(0, END), idx, one, END)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.isfinite(got[1]).all()
