"""Calls on a paged cache with more tokens, places and bytes a page than the small tests have: append with four tokens a workgroup and with
cu_new searched in memory, fork with more places than a workgroup has threads, pages that are copied in several pieces."""
import numpy as np
import pytest

import paper_2510_10620_amd as P
from oracle import paged as OP
from tests.test_gpu_paged import append, attend, check, ints, make_cache, mirror, randn, reserve, same_map, words

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,page,layout,hkv,d", [("bf16", 16, "token", 2, 64), ("f32", 5, "gaps", 3, 32), ("bf16", 64, "head", 1, 128)])
@pytest.mark.parametrize("new", [[1022, 0, 3], [1400, 1, 611, 0, 90], [1025], [1, 1, 1, 2001]])
def test_append_of_more_tokens_than_workgroups_take_one_by_one(dtype, page, layout, hkv, d, new):
    """1 025 tokens and more, no multiple of four among them; places that are padding or refused lie between."""
    rng = np.random.default_rng(len(new))
    lens = [int(x) for x in rng.integers(0, 3 * page, len(new))]
    cache, names = make_cache(lens, page, hkv, d, dtype, layers=2, spare=sum(-(-x // page) + 1 for x in new), width=-(-2100 // page) + 4, seed=page, layout=layout)
    m = mirror(cache)
    seqs = [int(s) for s in names] + [-1, int(names[0])]
    status = reserve(cache, m, seqs, new + [7, 1])
    assert status.tolist() == [OP.OK] * (len(new) + 1) + [OP.BAD]
    append(cache, m, seqs, new + [7, 1], status, 1, 5)
    same_map(cache, m)


def test_append_one_token_each_of_thousands_of_places():
    """More than 1 024 places without cu_new (four a workgroup), and with it, as counts of 0, 1 and 2."""
    import torch
    n, page = 2501, 4
    cache = P.Cache.empty(1, 4000, page, 1, 32, n + 3, 3, torch.bfloat16)
    cache.k.zero_()
    cache.v.zero_()
    m = mirror(cache)
    rng = np.random.default_rng(2)
    seqs = [int(s) for s in rng.permutation(n + 3)[:n]]
    seqs[7] = seqs[2000] = -1
    status = ints([7] * n)
    P.dcp_cache_reserve(cache, ints(seqs), status)
    k, v = randn((n, 1, 32), "bf16", 3), randn((n, 1, 32), "bf16", 4)
    P.dcp_cache_append(cache, k, v, seqs=ints(seqs), status=status)
    want, page_at = [], 0
    for i, s in enumerate(seqs):   # every place takes a page, in order, until none is left
        if s >= 0:
            m.table[s, 0], m.ref[page_at], m.length[s] = page_at, 1, 1
            m.k[0, page_at, 0], m.v[0, page_at, 0] = words(k)[i], words(v)[i]
            page_at += 1
        want.append(OP.OK)
    assert status.tolist() == want
    same_map(cache, m)
    new = [int(x) for x in rng.integers(0, 3, n)]
    P.dcp_cache_reserve(cache, ints(seqs), status, n_new=ints(new))
    for s, x in zip(seqs, new):    # still within the first page
        if s >= 0:
            m.length[s] += x
    assert status.tolist() == [OP.OK] * n
    append(cache, m, seqs, new, status, 0, 9)
    same_map(cache, m)


@pytest.mark.parametrize("pages", [4000, 500])
def test_fork_of_more_places_than_threads(pages):
    """1 500 places from a few sources; some are padding, name a sequence that does not exist, or a destination twice; with 500 pages they run out."""
    import torch
    rng = np.random.default_rng(pages)
    page, n, n_seqs = 4, 1500, 1700
    cache = P.Cache.empty(2, pages, page, 1, 32, n_seqs, 5, torch.bfloat16)
    cache.k.normal_()
    cache.v.normal_()
    m = mirror(cache)
    lens = [int(x) for x in rng.integers(0, 5 * page + 1, 20)]
    lens[3], lens[4] = 8, 0
    reserve(cache, m, list(range(20)), lens)
    src = [int(x) for x in rng.integers(0, 20, n)]
    dst = [20 + int(x) for x in rng.permutation(n_seqs - 20)[:n]]
    for i in range(0, n, 37):
        src[i] = -1 if i % 2 else n_seqs + 5
    dst[1200], dst[1300], dst[1400] = dst[10], n_seqs, 3
    status = ints([7] * n)
    P.dcp_cache_fork(cache, ints(src), ints(dst), status)
    torch.cuda.synchronize()
    want = m.fork(src, dst)
    assert status.tolist() == want and set(want) == ({OP.OK, OP.BAD} if pages == 4000 else {OP.OK, OP.FULL, OP.BAD})
    same_map(cache, m)


@pytest.mark.parametrize("dtype,page,hkv,d,layout", [("bf16", 37, 3, 128, "token"), ("bf16", 64, 8, 128, "gaps"), ("f32", 100, 2, 64, "head"), ("f32", 33, 5, 32, "token")])
def test_pages_of_several_pieces(dtype, page, hkv, d, layout):
    """Pages of more than 16 KiB, filled to one token, to the middle of a piece and to the brim, forked and moved; then read by attention."""
    import torch
    e = 2 if dtype == "bf16" else 4
    assert page * hkv * d * e > 1024 * 16
    lens = [1, page // 2, page - 1, page, 2 * page + 3, 3 * page - 1, 0]
    cache, names = make_cache(lens, page, hkv, d, dtype, layers=2, spare=8, extra_seqs=7, seed=page, layout=layout)
    m = mirror(cache)
    names = [int(s) for s in names]
    empty = [s for s in range(14) if s not in names]
    status = ints([7] * 7)
    P.dcp_cache_fork(cache, ints(names), ints(empty), status)
    torch.cuda.synchronize()
    assert status.tolist() == m.fork(names, empty) == [OP.OK] * 7
    same_map(cache, m)
    P.dcp_cache_free(cache, ints(names[:5]))
    m.free(names[:5])
    counts, ws = ints([0, 0]), torch.empty(P.dcp_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda").random_()
    P.dcp_cache_compact(cache, counts, ws)
    torch.cuda.synchronize()
    moved = m.compact()
    assert counts.tolist() == moved and moved[1] > 0
    same_map(cache, m)
    q = randn((7, 2 * hkv, d), dtype, 6)
    out, lse = attend(cache, q, 0.1, ints(empty))
    check(cache, q, out, lse, 0.1, empty)
