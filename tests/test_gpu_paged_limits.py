"""Calls on a paged cache at the ends of what they accept."""
import ctypes

import pytest

import paper_2510_10620_amd as P
from paper_2510_10620_amd import _lib
from tests.test_gpu_paged import NAN, attend, check, ints, make_cache, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages", [1 << 30, (1 << 30) - 1])
def test_needs_whose_sum_passes_31_bits(n_pages):
    """Two places that each want as many pages as a cache may have, of which three are free: neither is served, nothing changes."""
    import torch
    ref = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    ref[-3:] = 0
    table, length, kv = torch.empty((2, n_pages), dtype=torch.int32, device="cuda"), ints([0, 0]), torch.zeros(64, device="cuda")
    c = _lib.Cache()
    c.n_layers, c.n_pages, c.page_size, c.hkv, c.d, c.dtype, c.n_seqs, c.max_pages = 1, n_pages, 1, 1, 32, P.DCP_BF16, 2, n_pages
    for x in "kv":   # never followed here
        setattr(c, x, kv.data_ptr())
        for letter in "lpth":
            setattr(c, f"{x}_stride_{letter}", 32)
    c.page_ref, c.page_table, c.seq_len = ref.data_ptr(), table.data_ptr(), length.data_ptr()
    status, new, stream = ints([7, 7]), ints([n_pages, n_pages]), torch.cuda.current_stream().cuda_stream
    assert _lib.load().dcp_cache_reserve(ctypes.byref(c), None, new.data_ptr(), 2, status.data_ptr(), stream) == 0
    assert status.tolist() == [P.DCP_PLACE_FULL] * 2 and length.tolist() == [0, 0]
    assert int((ref == 0).sum()) == 3 and ref[-3:].tolist() == [0, 0, 0]
    # what is there goes to the first that asks for no more
    new.copy_(ints([3, n_pages]))
    assert _lib.load().dcp_cache_reserve(ctypes.byref(c), None, new.data_ptr(), 2, status.data_ptr(), stream) == 0
    assert status.tolist() == [P.DCP_PLACE_OK, P.DCP_PLACE_FULL] and length.tolist() == [3, 0]
    assert table[0, :3].tolist() == [n_pages - 3, n_pages - 2, n_pages - 1] and ref[-3:].tolist() == [1, 1, 1]


@pytest.mark.parametrize("lens", [[-1], [-5, 0, -(1 << 31)]])
def test_fork_into_sequences_of_negative_length(lens):
    """A length below 0 is cut to 0 in every call: such a sequence is empty, and may be forked into as it may be grown."""
    import torch
    cache = P.Cache.empty(2, 12, 8, 2, 32, 6, 3, torch.bfloat16)
    cache.k.normal_()
    cache.v.normal_()
    status = ints([7])
    P.dcp_cache_reserve(cache, ints([5]), status, n_new=ints([11]))
    for i, n in enumerate(lens):
        cache.seq_len[i] = n
    status = ints([7] * len(lens))
    P.dcp_cache_fork(cache, ints([5] * len(lens)), ints(range(len(lens))), status)
    assert status.tolist() == [P.DCP_PLACE_OK] * len(lens)
    assert cache.seq_len.tolist() == [11] * len(lens) + [0] * (5 - len(lens)) + [11]
    pages = cache.page_table.cpu()
    for i in range(len(lens)):
        assert pages[i, 0] == pages[5, 0] == 0 and pages[i, 1] == 2 + i
        assert torch.equal(cache.k[:, 2 + i, :3], cache.k[:, 1, :3]) and torch.equal(cache.v[:, 2 + i, :3], cache.v[:, 1, :3])
    assert cache.page_ref.tolist() == [1 + len(lens), 1] + [1] * len(lens) + [0] * (10 - len(lens))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["beside", "halves", "heads first", "other heads"])
def test_queries_and_outputs_in_one_buffer(dtype, layout):
    """Outputs that lie between the queries of one buffer, and that overlap them by one row."""
    import torch
    n, hq, d = 5, 4, 64
    cache, names = make_cache([70, 1, 333, 16, 0], 32, 2, d, dtype, seed=5)
    places = [int(s) for s in names]
    rand = randn((n, 2, hq, d), dtype, 6)
    if layout == "beside":          # [n, 2, hq, d]: a token's queries, then its outputs
        q, out = rand[:, 0], rand[:, 1]
        bad = rand.view(n, 2 * hq, d)[:, 1: hq + 1]
    elif layout == "halves":        # [n, hq, 2 d]: a head's query, then its output
        both = rand.view(n, hq, 2 * d)
        q, out = both[:, :, :d], both[:, :, d:]
        bad = both[:, :, d // 2: d // 2 + d]
    elif layout == "heads first":   # [2 hq, n, d]
        both = rand.view(2 * hq, n, d).transpose(0, 1)
        q, out = both[:, :hq], both[:, hq:]
        bad = both[:, 1: hq + 1]
    else:                           # every other head
        both = rand.view(n, 2 * hq, d)
        q, out = both[:, ::2], both[:, 1::2]
        bad = q
    kept = q.clone()
    out.fill_(NAN)
    lse, ws = torch.full((hq, n), NAN, device="cuda"), torch.empty(P.dcp_paged_attn_workspace_bytes(cache, n, hq), dtype=torch.uint8, device="cuda")
    P.dcp_paged_attn_fwd(cache, q, out, lse, 0.1, ws, seqs=ints(names))
    torch.cuda.synchronize()
    assert torch.equal(q, kept)
    check(cache, kept, out, lse, 0.1, places)
    want, want_l = attend(cache, kept, 0.1, ints(names))
    assert torch.equal(out, want) and torch.equal(lse, want_l)
    with pytest.raises(P.DcpError) as ei:
        P.dcp_paged_attn_fwd(cache, q, bad, lse, 0.1, ws, seqs=ints(names))
    assert ei.value.status == P.DCP_ERR_INVALID_ARG and "overlaps" in str(ei.value)
