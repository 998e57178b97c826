"""Attention of the last tokens of every place over a paged key-value cache in 8 bits against the 64-bit oracle.  Rows that no place has, and slots
without a token, hold NaN."""
import numpy as np
import pytest

import paper_2510_10620_amd as P
from oracle import e4m3
from oracle import paged as OP
from tests.paged8 import NAN, Held, check_rows, dtype_of, f64, infinite_at, ints, make_cache, randn

pytestmark = pytest.mark.gpu

# bf16 weights are rounded once, to half a step of 2^-8 at most; that is a relative error of each, and so of their sum over |v|
WEIGHTS = 2.0 ** -8


# Few rows, of a place or of the whole batch, are walked with the keys in registers, more with the keys in LDS.
BOTH = pytest.mark.parametrize("in_lds", [False, True])


def behind(n, hq, hkv):
    """Rows behind those of the places, which no place has, with which a batch counts as one of many rows."""
    return 1024 // hq + 24 * n * hkv // hq + 2


def chunk(cache, q, scale, cu, seqs=None, window=0, sink=0, layer=0, status=None, ws=None, in_lds=False):
    import torch
    if in_lds:
        t, more = q.shape[0], behind(len(cu) - 1, q.shape[1], cache.k.shape[3])
        out, lse = chunk(cache, torch.cat([q, torch.full((more, *q.shape[1:]), NAN, dtype=q.dtype, device="cuda")]), scale, cu, seqs, window, sink, layer, status)
        assert bool(torch.isnan(out[t:]).all()) and bool(torch.isnan(lse[:, t:]).all())
        return out[:t].contiguous(), lse[:, :t].contiguous()
    out, lse = torch.full_like(q, NAN), torch.full((q.shape[1], q.shape[0]), NAN, dtype=torch.float32, device="cuda")
    if ws is None:
        ws = torch.empty(P.dcp_paged_attn_chunk_workspace_bytes(cache, len(cu) - 1, q.shape[0], q.shape[1]), dtype=torch.uint8, device="cuda").random_()
    P.dcp_paged_attn_chunk_fwd(cache, q, out, lse, scale, ws, ints(cu), seqs=seqs, window=window, sink=sink, layer=layer, status=status)
    torch.cuda.synchronize()
    return out, lse


def rows_of(length, places, cu, tokens):
    """(row, sequence, position) of the rows that exist"""
    return [(t, s, int(length[s]) - cu[i + 1] + t) for i, s in enumerate(places) if 0 <= s < len(length)
            for t in range(cu[i], min(cu[i + 1], tokens)) if int(length[s]) - cu[i + 1] + t >= 0]


def batch(lens, new, names, pad=1):
    places = [int(s) for s in names] + [-1] * pad
    return places, np.concatenate([[0], np.cumsum(list(new) + [0] * pad)]).tolist()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 32])
@pytest.mark.parametrize("page,block", [(1, 1), (16, 16), (20, 10), (37, 37), (64, 8), (256, 64)])
def test_lengths_pages_and_blocks(io, d, page, block):
    lens = [0, 1, 2, 31, 33, 63, 64, 65, 100, 129, 200, 300]
    new = [3, 1, 2, 31, 1, 40, 64, 65, 2, 130, 0, 33]     # more than there are in the first and the tenth
    cache, names = make_cache(lens, page, block, 2, d, io, seed=page)
    places, cu = batch(lens, new, names)
    q = randn((cu[-1] + 2, 6, d), io, 1)
    out, lse = chunk(cache, q, d ** -0.5, cu, ints(places))
    check_rows(cache, q, out, lse, d ** -0.5, rows_of(cache.seq_len.tolist(), places, cu, q.shape[0]), weights=WEIGHTS)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 32])
@pytest.mark.parametrize("page,block", [(1, 1), (8, 8), (16, 16), (20, 10), (24, 8), (37, 37), (64, 4), (256, 64)])
@pytest.mark.parametrize("hq", [4, 8])
def test_few_tokens(io, d, page, block, hq):
    """Up to 24 rows of a place and KV head on average (hq 4: 13), and some more (hq 8: 25); one place has many."""
    lens = [0, 1, 2, 31, 33, 63, 64, 65, 100, 129, 200, 300, 1000, 77, 78, 5, 4, 3]
    new = [3, 1, 2, 5, 1, 4, 8, 7, 60, 8, 0, 6, 3, 1, 1, 5, 1, 3]
    cache, names = make_cache(lens, page, block, 2, d, io, seed=page)
    places, cu = batch(lens, new, names)
    q = randn((cu[-1] + 2, hq, d), io, 1)
    out, lse = chunk(cache, q, d ** -0.5, cu, ints(places))
    check_rows(cache, q, out, lse, d ** -0.5, rows_of(cache.seq_len.tolist(), places, cu, q.shape[0]), weights=WEIGHTS)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (4, 1), (6, 2), (7, 1), (16, 1), (40, 1), (64, 2), (130, 1), (24, 8)])
@BOTH
def test_heads(io, hq, hkv, in_lds):
    lens, new = [5, 300, 64], [5, 17, 3]
    cache, names = make_cache(lens, 16, 16, hkv, 64, io, seed=hq)
    places, cu = batch(lens, new, names)
    q = randn((cu[-1], hq, 64), io, 2)
    out, lse = chunk(cache, q, 0.125, cu, ints(places), in_lds=in_lds)
    check_rows(cache, q, out, lse, 0.125, rows_of(cache.seq_len.tolist(), places, cu, cu[-1]), weights=WEIGHTS)


@pytest.mark.parametrize("io,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (5, 3), (16, 40), (64, 0), (100, 64), (33, 31), (5000, 7), (2 ** 31 - 1, 2 ** 31 - 1), (0, 9)])
@pytest.mark.parametrize("new", [[1, 20, 9, 100, 80], [1, 5, 9, 4, 6]])
@BOTH
def test_window_and_sink(io, d, window, sink, new, in_lds):
    lens = [1, 20, 64, 130, 700]
    cache, names = make_cache(lens, 32, 16, 2, d, io)
    places, cu = batch(lens, new, names)
    q = randn((cu[-1], 4, d), io, 3)
    out, lse = chunk(cache, q, d ** -0.5, cu, ints(places), window=window, sink=sink, in_lds=in_lds)
    check_rows(cache, q, out, lse, d ** -0.5, rows_of(cache.seq_len.tolist(), places, cu, cu[-1]), window, sink, weights=WEIGHTS)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["token", "head", "gaps", "mixed"])
@pytest.mark.parametrize("new", [[30, 90, 3], [30, 40, 3], [3, 4, 1]])
def test_layouts_layers_and_strides(io, layout, new):
    import torch
    lens = [40, 333, 3]
    cache, names = make_cache(lens, 16, 8, 3, 64, io, layers=3, layout=layout)
    places, cu = batch(lens, new, names)
    q = randn((cu[-1], 9, 72), io, 4)[:, :, :64]
    rows = rows_of(cache.seq_len.tolist(), places, cu, cu[-1])
    for layer in (0, 2):
        out, lse = torch.full((9, cu[-1], 80), NAN, dtype=q.dtype, device="cuda").transpose(0, 1)[:, :, :64], torch.full((9, cu[-1]), NAN, device="cuda")
        ws = torch.empty(P.dcp_paged_attn_chunk_workspace_bytes(cache, len(places), cu[-1], 9), dtype=torch.uint8, device="cuda")
        P.dcp_paged_attn_chunk_fwd(cache, q, out, lse, 0.2, ws, ints(cu), seqs=ints(places), layer=layer)
        check_rows(cache, q, out, lse, 0.2, rows, layer=layer, weights=WEIGHTS)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@BOTH
def test_large_scores_and_far_away_maxima(io, in_lds):
    import torch
    cache, names = make_cache([900], 64, 16, 1, 128, io)
    cache.k_scale[:, cache.page_table[int(names[0])][::2].long()] += 4
    q = randn((200, 2, 128), io, 5, 3.0)
    out, lse = chunk(cache, q, 0.3, [0, 200], ints(names), in_lds=in_lds)
    check_rows(cache, q, out, lse, 0.3, rows_of(cache.seq_len.tolist(), [int(names[0])], [0, 200], 200), weights=WEIGHTS)


def test_one_token_is_the_other_entry_point():
    import torch
    lens = [0, 1, 64, 65, 700, 3000]
    cache, names = make_cache(lens, 32, 32, 2, 128)
    q = randn((6, 8, 128), "bf16", 6)
    out, lse = chunk(cache, q, 0.1, list(range(7)), ints(names))
    o2, l2 = torch.full_like(out, NAN), torch.full_like(lse, NAN)
    ws = torch.empty(P.dcp_paged_attn_workspace_bytes(cache, 6, 8), dtype=torch.uint8, device="cuda")
    P.dcp_paged_attn_fwd(cache, q, o2, l2, 0.1, ws, seqs=ints(names))
    held = Held(cache)
    rows = [(i, int(s), n - 1) for i, (s, n) in enumerate(zip(names, lens)) if n]
    check_rows(cache, q, out, lse, 0.1, rows, weights=WEIGHTS, held=held)
    o2[0], l2[:, 0] = NAN, NAN          # an empty sequence: O = 0 there, no row here
    check_rows(cache, q, o2, l2, 0.1, rows, held=held)


def test_status_pages_and_rows_that_do_not_exist():
    lens, new = [100, 100, 100, 64, 50], [20, 30, 10, 5, 40]
    cache, names = make_cache(lens, 16, 16, 2, 128)
    a, b, c, d, e = (int(s) for s in names)
    cache.page_table[a, 1], cache.page_table[a, 5], cache.page_table[b, :] = -1, 10 ** 6, -5
    places, cu = [a, b, c, d, e, 1000], [4] + (4 + np.cumsum(new + [3])).tolist()
    q = randn((cu[5] - 7, 8, 128), "bf16", 7)               # the last rows of e are not there
    out, lse = chunk(cache, q, 0.1, cu, ints(places), status=ints([0, 0, 1, 0, 0, 0]))
    rows = rows_of([int(x) if s != c else 0 for s, x in enumerate(cache.seq_len.tolist())], places, cu, q.shape[0])
    check_rows(cache, q, out, lse, 0.1, rows, weights=WEIGHTS)


@pytest.mark.parametrize("io,d", [("bf16", 128), ("bf16", 32), ("f32", 64)])
@pytest.mark.parametrize("page,block", [(16, 16), (20, 5)])
@pytest.mark.parametrize("shared", [False, True])
def test_few_tokens_nan_and_infinity_reach_who_sees_them(io, d, page, block, shared):
    """shared: a sequence so long that several workgroups walk it."""
    import torch
    n = 5000 if shared else 200
    cache, names = make_cache([n] * 3, page, block, 1, d, io)
    k, v = cache.k.view(torch.uint8), cache.v.view(torch.uint8)
    where = lambda i, pos: (0, int(cache.page_table[int(names[i]), pos // page]), pos % page, 0)   # noqa: E731
    v[(*where(0, n - 4), 7)] = 0x7f           # seen by the last four of eight tokens
    v[(*where(0, n - 90), 8)] = 0xff          # and by all
    k[(*where(1, n - 3), 5)] = 0x7f
    at = where(2, n - 2)
    cache.v_scale[0, at[1], at[2] // block] = 250
    for pos in range(n - 2 - (n - 2) % page % block, n):
        if where(2, pos)[1] == at[1] and where(2, pos)[2] // block == at[2] // block:
            v[where(2, pos)] = 0
    v[(*at, 3)], v[(*at, 4)], v[(*at, 5)] = 0x60, 0xe8, 0x08   # 2^5 and -2^6 times 2^123: infinities; 2^-6 times it
    places, cu = batch([n] * 3, [8] * 3, names, 0)
    q = randn((24, 4, d), io, 8)
    out, lse = chunk(cache, q, d ** -0.5, cu, ints(places))
    o, l = f64(out).reshape(3, 8, 4, d), f64(lse).T.reshape(3, 8, 4)
    assert np.isnan(o[0, 4:, :, 7]).all() and np.isfinite(o[0, :4, :, 7]).all() and np.isnan(o[0, :, :, 8]).all() and np.isfinite(l[0]).all()
    assert np.isfinite(np.delete(o[0], [7, 8], 2)).all()
    assert np.isnan(o[1, 5:]).all() and np.isnan(l[1, 5:]).all() and np.isfinite(o[1, :5]).all() and np.isfinite(l[1, :5]).all()
    assert np.isfinite(o[2, :6]).all() and (o[2, 6:, :, 3] == np.inf).all() and (o[2, 6:, :, 4] == -np.inf).all()
    assert np.isfinite(o[2, 6:, :, 5]).all() and (np.abs(o[2, 6:, :, 5]) > 1e25).all()


@pytest.mark.parametrize("io,d", [("bf16", 128), ("bf16", 32), ("f32", 64)])
@BOTH
def test_nan_and_infinity_reach_who_sees_them(io, d, in_lds):
    import torch
    cache, names = make_cache([200, 200, 200, 200], 16, 16, 1, d, io)
    row = {i: cache.page_table[int(s)].tolist() for i, s in enumerate(names)}
    k, v = cache.k.view(torch.uint8), cache.v.view(torch.uint8)
    v[0, row[0][11], 9, 0, 7] = 0x7f        # place 0: V of token 185, number 7
    k[0, row[1][11], 3, 0, 5] = 0xff        # place 1: K of token 179
    v[0, row[2][12], 8:, :, :] = 0x7f       # place 2: behind the last token
    # place 3: token 187 stands for infinities in its number 3, -infinities in 4 and both with 190 in 5
    cache.v_scale[0, row[3][11]] = 247
    v[0, row[3][11], :, 0, :] = 0
    v[0, row[3][11], 11, 0, 3], v[0, row[3][11], 11, 0, 4], v[0, row[3][11], 11, 0, 5], v[0, row[3][11], 14, 0, 5] = 0x7e, 0xfe, 0x7e, 0xfe
    places, cu = batch([200] * 4, [40] * 4, names, 0)
    q = randn((160, 4, d), io, 8)
    q[125, 2, 5] = NAN                      # place 3, one row
    out, lse = chunk(cache, q, d ** -0.5, cu, ints(places), in_lds=in_lds)
    o, l = f64(out), f64(lse)
    at = lambda i: o[40 * i: 40 * i + 40]   # noqa: E731
    assert np.isnan(at(0)[25:, :, 7]).all() and np.isfinite(at(0)[:25]).all() and np.isfinite(np.delete(at(0), 7, 2)).all() and np.isfinite(l[:, :40]).all()
    assert np.isnan(at(1)[19:]).all() and np.isfinite(at(1)[:19]).all()
    assert np.isfinite(at(2)).all()
    x = at(3)
    assert np.isnan(x[5, 2]).all()
    x[5, 2] = x[5, 1]
    assert np.isfinite(np.delete(x, [3, 4, 5], 2)).all() and np.isfinite(x[:27]).all()
    assert (x[27:, :, 3] == np.inf).all() and (x[27:, :, 4] == -np.inf).all()
    assert (x[27:30, :, 5] == np.inf).all() and np.isnan(x[30:, :, 5]).all()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 32])
@pytest.mark.parametrize("n", [150, 5000])
@BOTH
def test_infinite_keys_and_values_that_all_see(io, d, n, in_lds):
    """With queries of few bits, whose lower parts are zero, as are those of a weight of one."""
    import torch
    cache, names = make_cache([n, n], 16, 16, 1, d, io)
    k, v = cache.k.view(torch.uint8), cache.v.view(torch.uint8)
    a, b = (int(s) for s in names)
    k[0, cache.page_table[a].long()] = 0                       # every key weighs the same
    p, slot = infinite_at(cache, a, 20)
    k[0, p, slot] = 0
    p, slot = infinite_at(cache, b, 20)
    v[0, p, slot] = 0
    q = randn((10, 4, d), io, 1)
    q[5:, :, 5] = -1.0
    out, lse = chunk(cache, q, 0.1, [0, 5, 10], ints(names), in_lds=in_lds)
    o = f64(out)
    assert (o[:5, :, 3] == np.inf).all() and (o[:5, :, 4] == -np.inf).all() and np.isfinite(np.delete(o[:5], [3, 4], 2)).all()
    # a score of -inf weighs what -2^127 weighs
    cache.k_scale[0, p, slot // 16] = 245
    o2, l2 = chunk(cache, q, 0.1, [0, 5, 10], ints(names), in_lds=in_lds)
    assert np.isfinite(o[5:]).all() and np.isfinite(f64(lse)[:, 5:]).all() and torch.equal(out[5:], o2[5:]) and torch.equal(lse[:, 5:], l2[:, 5:])
    cache.k_scale[0, p, slot // 16] = 247
    q[5:, :, 5] = 1.0
    out, lse = chunk(cache, q, 0.1, [0, 5, 10], ints(names), in_lds=in_lds)
    assert np.isnan(f64(out)[5:]).all()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[3, 40, 70, 300], [3, 4, 7, 3]])
def test_items_that_many_workgroups_share(io, new):
    lens = [9000, 40, 5000, 700]
    cache, names = make_cache(lens, 64, 64, 2, 128, io)
    places, cu = batch(lens, new, names)
    q = randn((cu[-1], 8, 128), io, 9)
    rows = rows_of(cache.seq_len.tolist(), places, cu, cu[-1])
    out, lse = chunk(cache, q, 0.088, cu, ints(places))
    some = rows[::7]
    import torch
    keep = torch.zeros(cu[-1], dtype=torch.bool, device="cuda")
    keep[[r for r, _, _ in some]] = True
    assert not torch.isnan(out).any() and not torch.isnan(lse).any()
    out[~keep], lse[:, ~keep] = NAN, NAN
    check_rows(cache, q, out, lse, 0.088, some, weights=WEIGHTS)


@pytest.mark.parametrize("new", [40, 5])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_nan_in_items_that_one_workgroup_has_whole(io, new):
    """So many items that most are walked by one workgroup, from the first key tile to the last."""
    import torch
    places, d, hkv = 64, 64, 8
    cache, names = make_cache([200] * places, 16, 16, hkv, d, io)
    v, length = cache.v.view(torch.uint8), 200
    pages = cache.page_table[torch.from_numpy(np.asarray(names)).cuda().long()]
    v[0, pages[:, (length - 3) // 16].long(), (length - 3) % 16, :, 7] = 0x7f
    q = randn((places * new, 4 * hkv, d), io, 8)
    out, lse = chunk(cache, q, d ** -0.5, [new * i for i in range(places + 1)], ints(names))
    o = f64(out).reshape(places, new, 4 * hkv, d)
    assert np.isnan(o[:, new - 3:, :, 7]).all() and np.isfinite(o[:, : new - 3]).all() and np.isfinite(np.delete(o, 7, 3)).all() and np.isfinite(f64(lse)).all()
    # what is finite is what it is without the NaN
    v[0, pages[:, (length - 3) // 16].long(), (length - 3) % 16, :, 7] = 0
    clean, _ = chunk(cache, q, d ** -0.5, [new * i for i in range(places + 1)], ints(names))
    c = f64(clean).reshape(places, new, 4 * hkv, d)
    assert np.array_equal(np.delete(c, 7, 3), np.delete(o, 7, 3)) and np.array_equal(c[:, : new - 3], o[:, : new - 3])


@BOTH
def test_a_sequence_in_several_places(in_lds):
    cache, names = make_cache([300, 50], 16, 16, 2, 64)
    a, b = (int(s) for s in names)
    places, cu = [a, b, a, a], [0, 40, 50, 51, 60]
    q = randn((60, 4, 64), "bf16", 3)
    out, lse = chunk(cache, q, 0.125, cu, ints(places), in_lds=in_lds)
    check_rows(cache, q, out, lse, 0.125, rows_of(cache.seq_len.tolist(), places, cu, 60), weights=WEIGHTS)


def test_binding_refuses():
    import torch
    cache, names = make_cache([30, 20], 16, 8, 2, 64)
    q = randn((5, 4, 64), "bf16", 1)
    out, lse, cu = torch.empty_like(q), torch.empty((4, 5), device="cuda"), ints([0, 3, 5])
    ws = torch.empty(P.dcp_paged_attn_chunk_workspace_bytes(cache, 2, 5, 4), dtype=torch.uint8, device="cuda")
    good = dict(q=q, out=out, lse=lse, softmax_scale=0.1, workspace=ws, cu_new=cu, seqs=ints(names))
    P.dcp_paged_attn_chunk_fwd(cache, **good)
    for bad in (dict(q=q.float()), dict(out=out[:4]), dict(lse=lse[:, :4]), dict(lse=lse.double()), dict(lse=torch.empty((5, 4), device="cuda").t()),
                dict(cu_new=cu.long()), dict(cu_new=cu.cpu()), dict(seqs=ints([1])), dict(q=q[:, :, ::2]), dict(workspace=ws.cpu()), dict(status=ints([0]))):
        with pytest.raises(Exception):
            P.dcp_paged_attn_chunk_fwd(cache, **dict(good, **bad))
    k = torch.empty((5, 2, 64), dtype=torch.bfloat16, device="cuda")
    for a, b in ((k.float(), k.float()), (k, k[:4]), (k[:, :1], k[:, :1]), (k.cpu(), k), (k, k)):
        with pytest.raises(Exception):
            P.dcp_cache_read(cache, a, b, cu_new=ints([0, 5]))
    # caches
    e4m3fn, scales = torch.float8_e4m3fn, torch.zeros((1, 4, 2, 2), dtype=torch.uint8, device="cuda")
    kv = torch.zeros((1, 4, 16, 2, 64), dtype=torch.uint8, device="cuda").view(e4m3fn)
    ref, table, length = ints([0] * 4), ints([-1] * 6).view(2, 3), ints([0, 0])
    P.Cache(kv, kv, ref, table, length, k_scale=scales, v_scale=scales)
    for kw in (dict(), dict(k_scale=scales), dict(k_scale=scales, v_scale=scales[:, :, :1]), dict(k_scale=scales.float(), v_scale=scales.float()),
               dict(k_scale=scales.cpu(), v_scale=scales.cpu()), dict(k_scale=scales.repeat(1, 1, 2, 1)[:, :, :3].contiguous(), v_scale=scales.repeat(1, 1, 2, 1)[:, :, :3].contiguous()),
               dict(k_scale=scales, v_scale=scales.transpose(2, 3)), dict(k_scale=scales[:, :3].contiguous(), v_scale=scales[:, :3].contiguous())):
        with pytest.raises(ValueError):
            P.Cache(kv, kv, ref, table, length, **kw)
    with pytest.raises(TypeError):
        P.Cache(kv, kv, ref, table, length, k_scale=scales, v_scale=scales, io_dtype=torch.float16)
    half = kv.view(torch.uint8).to(torch.bfloat16)
    for kw in (dict(k_scale=scales), dict(io_dtype=torch.float32)):
        with pytest.raises(ValueError):
            P.Cache(half, half, ref, table, length, **kw)
    with pytest.raises(ValueError):
        P.Cache.empty(1, 4, 16, 2, 64, 2, 3, e4m3fn, scale_block=5)
    with pytest.raises(ValueError):
        P.Cache.empty(1, 4, 16, 2, 64, 2, 3, torch.bfloat16, scale_block=16)
    other = P.Cache.empty(1, 4, 16, 2, 64, 2, 3, torch.bfloat16)
    with pytest.raises(Exception, match="dcp_block_attn_fwd"):
        P.dcp_paged_attn_chunk_fwd(other, **good)


def test_thousands_of_places():
    lens = [1 + i % 5 for i in range(3000)]
    cache, names = make_cache(lens, 4, 4, 1, 32)
    new = [1 + i % 3 for i in range(3000)]
    places, cu = batch(lens, new, names)
    q = randn((cu[-1], 2, 32), "bf16", 10)
    out, lse = chunk(cache, q, 0.2, cu, ints(places))
    check_rows(cache, q, out, lse, 0.2, rows_of(cache.seq_len.tolist(), places, cu, cu[-1]), weights=WEIGHTS)


@pytest.mark.parametrize("io,window", [("bf16", 0), ("f32", 70)])
def test_few_tokens_in_batches_padded_to_any_size(io, window):
    """Few items are listed by the walk itself, more by a launch before it: the shares, and so the bits, are the same."""
    lens, new = [3 + 53 * i % 700 for i in range(40)], [1 + i % 5 for i in range(40)]
    lens = [n + m for n, m in zip(lens, new)]
    cache, names = make_cache(lens, 16, 16, 2, 64, io, seed=3)
    q = randn((sum(new), 8, 64), io, 1)
    seen = []
    for pad in (0, 150, 180, 220, 260, 1500):   # 480 rows are 30 items of 16, and one more a place: 70 to 1 570 items at most
        places, cu = batch(lens, new, names, pad)
        out, lse = chunk(cache, q, 0.125, cu, seqs=ints(places), window=window)
        if not seen:
            check_rows(cache, q, out, lse, 0.125, rows_of(cache.seq_len.tolist(), places, cu, cu[-1]), window=window)
        seen.append((f64(out), f64(lse)))
        assert np.array_equal(seen[0][0], seen[-1][0]) and np.array_equal(seen[0][1], seen[-1][1])


def test_begins_that_are_not_ascending_stay_inside():
    """What the rows get is not said; nothing outside q, out and lse is touched, and the call ends."""
    import torch
    cache, names = make_cache([300, 300, 300], 16, 16, 2, 64)
    q = randn((300, 4, 64), "bf16", 11)
    room = torch.full((3, 300, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((3, 4, 300), 7.0, device="cuda")
    for cu in ([50, 10, 300, 2], [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1], [0, 300, 0, 300]):
        ws = torch.empty(P.dcp_paged_attn_chunk_workspace_bytes(cache, 3, 300, 4), dtype=torch.uint8, device="cuda")
        P.dcp_paged_attn_chunk_fwd(cache, q, room[1], lse[1], 0.1, ws, ints(cu), seqs=ints(names))
        torch.cuda.synchronize()
    assert bool((room[0] == 7).all()) and bool((room[2] == 7).all()) and bool((lse[0] == 7).all()) and bool((lse[2] == 7).all())


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_few_tokens_with_begins_that_are_not_ascending_stay_inside(io):
    """As above, with the items of 16 rows: places that name more rows between them than there are."""
    import torch
    cache, names = make_cache([300, 300, 300, 5, 0, 90], 16, 16, 2, 64, io)
    q = randn((64, 4, 64), io, 11)
    room = torch.full((3, 64, 4, 64), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((3, 4, 64), 7.0, device="cuda")
    for cu in ([50, 10, 64, 2, 64, 0, 64], [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0, 64, -5], [0, 64, 0, 64, 0, 64, 0], [64, 0, 0, 0, 0, 0, 0]):
        ws = torch.empty(P.dcp_paged_attn_chunk_workspace_bytes(cache, 6, 64, 4), dtype=torch.uint8, device="cuda")
        P.dcp_paged_attn_chunk_fwd(cache, q, room[1], lse[1], 0.1, ws, ints(cu), seqs=ints(names))
        torch.cuda.synchronize()
    assert bool((room[0] == 7).all()) and bool((room[2] == 7).all()) and bool((lse[0] == 7).all()) and bool((lse[2] == 7).all())


# ------------------------------------------------------------------------------------------------- as they are used
@pytest.mark.parametrize("io,d,window,sink", [("bf16", 128, 0, 0), ("bf16", 64, 24, 4), ("f32", 32, 0, 0)])
@pytest.mark.parametrize("graph", [False, True])
def test_prompt_in_pieces_drafts_and_single_tokens(io, d, window, sink, graph):
    """A prompt in two pieces, drafted tokens that are verified, then tokens one by one, for several layers; every step against the oracle, whose cache
    takes the same steps.  graph: a step of each kind is recorded once and replayed."""
    import torch
    layers, hkv, hq, page, block, scale = 2, 2, 6, 16, 8, d ** -0.5
    cache = P.Cache.empty(layers, 40, page, hkv, d, 4, 16, torch.float8_e4m3fn, scale_block=block, io_dtype=dtype_of(io))
    held = Held(cache)
    seqs = [2, 0, -1, 3]
    sizes = [[37, 5, 0, 20], [30, 61, 0, 1], [4, 4, 0, 4], [4, 4, 0, 4], [1, 1, 0, 1], [1, 1, 0, 1], [1, 1, 0, 1]]
    recorded = {}
    for step, new in enumerate(sizes):
        cu = np.concatenate([[0], np.cumsum(new)])
        single = max(new) == 1 and step >= 4
        tokens = 4 if single else int(cu[-1])
        key = tuple(new)
        if key not in recorded:
            s = dict(k=torch.empty((layers, tokens, hkv, d), dtype=dtype_of(io), device="cuda"), status=ints([0] * 4), n_new=ints(new), cu=ints(cu), seqs=ints(seqs))
            s.update(v=torch.empty_like(s["k"]), q=torch.empty((layers, tokens, hq, d), dtype=dtype_of(io), device="cuda"))
            s.update(out=torch.empty_like(s["q"]), lse=torch.empty((layers, hq, tokens), device="cuda"))
            size = P.dcp_paged_attn_workspace_bytes(cache, 4, hq) if single else P.dcp_paged_attn_chunk_workspace_bytes(cache, 4, tokens, hq)
            s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")

            def go(s=s, single=single):
                P.dcp_cache_reserve(cache, s["seqs"], s["status"], n_new=None if single else s["n_new"])
                for layer in range(layers):
                    if single:
                        P.dcp_cache_append(cache, s["k"][layer], s["v"][layer], seqs=s["seqs"], status=s["status"], layer=layer)
                        P.dcp_paged_attn_fwd(cache, s["q"][layer], s["out"][layer], s["lse"][layer], scale, s["ws"], seqs=s["seqs"], window=window, sink=sink,
                                             layer=layer, status=s["status"])
                    else:
                        P.dcp_cache_append(cache, s["k"][layer], s["v"][layer], seqs=s["seqs"], cu_new=s["cu"], status=s["status"], layer=layer)
                        P.dcp_paged_attn_chunk_fwd(cache, s["q"][layer], s["out"][layer], s["lse"][layer], scale, s["ws"], s["cu"], seqs=s["seqs"], window=window,
                                                   sink=sink, layer=layer, status=s["status"])
            s["go"] = go
            if graph:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    go()
                s["go"] = g.replay
            recorded[key] = s
        s = recorded[key]
        for name, seed in (("k", 1), ("v", 2), ("q", 3)):
            s[name].copy_(randn(s[name].shape, io, 10 * step + seed))
        s["out"].fill_(NAN)
        s["lse"].fill_(NAN)
        s["go"]()
        torch.cuda.synchronize()
        m = held.map()
        assert s["status"].tolist() == m.reserve(seqs, [1, 1, 1, 1] if single else new) == [0] * 4
        places_cu = list(range(5)) if single else cu.tolist()
        for layer in range(layers):
            e4m3.append(m, held.ks, held.vs, block, seqs, places_cu, f64(s["k"][layer]), f64(s["v"][layer]), [0] * 4, layer)
            check_rows(cache, s["q"][layer], s["out"][layer], s["lse"][layer], scale, rows_of(held.length, seqs, places_cu, tokens), window, sink, layer,
                       2.0 ** -15 if single else WEIGHTS, held)
        torch.empty(1000, device="cuda").normal_().sum().item()    # other work between replays


def test_two_streams_and_two_graphs_that_share_a_workspace():
    import torch
    lens, new = [500, 70, 1300], [33, 70, 9]
    caches = [make_cache(lens, 32, 16, 2, 64, seed=s) for s in (1, 2)]
    q = [randn((112, 4, 64), "bf16", s) for s in (3, 4)]
    batches = [batch(lens, new, names) for _, names in caches]
    want = [chunk(c, x, 0.125, cu, ints(places)) for (c, _), x, (places, cu) in zip(caches, q, batches)]
    size = P.dcp_paged_attn_chunk_workspace_bytes(caches[0][0], 4, 112, 4)

    def call(i, out, lse, ws, cu, seqs):
        P.dcp_paged_attn_chunk_fwd(caches[i][0], q[i], out, lse, 0.125, ws, cu, seqs=seqs)
    got = [(torch.full_like(q[i], NAN), torch.full_like(want[i][1], NAN)) for i in range(2)]
    args = [(ints(cu), ints(places)) for places, cu in batches]
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                call(i, *got[i], spaces[i], *args[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(got[i][0], want[i][0]) and torch.equal(got[i][1], want[i][1])
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i, *got[i], spaces[0], *args[i])
        graphs.append(g)
    for order in ((0, 1), (1, 0, 1), (0, 0, 1)):
        for i in range(2):
            got[i][0].fill_(NAN)
            got[i][1].fill_(NAN)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(got[i][0], want[i][0]) and torch.equal(got[i][1], want[i][1])
