"""A paged key-value cache in 8 bits: new tokens rounded into it, tokens read back, the attention of one new token, and the calls that move
pages, against the 64-bit oracle.  Slots without a token hold NaN, blocks without one bytes that are no scales."""
import numpy as np
import pytest

import paper_2510_10620_amd as P
from oracle import e4m3
from tests.paged8 import NAN, Held, check_rows, dtype_of, f64, infinite_at, ints, make_cache, randn

pytestmark = pytest.mark.gpu


def attend(cache, q, scale, seqs=None, window=0, sink=0, layer=0, status=None):
    import torch
    out, lse = torch.full_like(q, NAN), torch.full((q.shape[1], q.shape[0]), NAN, dtype=torch.float32, device="cuda")
    ws = torch.empty(P.dcp_paged_attn_workspace_bytes(cache, q.shape[0], q.shape[1]), dtype=torch.uint8, device="cuda").random_()
    P.dcp_paged_attn_fwd(cache, q, out, lse, scale, ws, seqs=seqs, window=window, sink=sink, layer=layer, status=status)
    torch.cuda.synchronize()
    return out, lse


def last_tokens(cache, places):
    length = cache.seq_len.tolist()
    return [(i, s, length[s] - 1) for i, s in enumerate(places) if 0 <= s < len(length)]


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 400, 1000]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 32])
@pytest.mark.parametrize("page,block", [(1, 1), (8, 4), (16, 16), (20, 10), (37, 37), (64, 1), (64, 16), (64, 64), (96, 48)])
def test_attend_lengths_pages_and_blocks(io, d, page, block):
    cache, names = make_cache(EDGES, page, block, 2, d, io, seed=page)
    places = [int(s) for s in names] + [-1, 1000]
    q = randn((len(places), 8, d), io, 1)
    out, lse = attend(cache, q, d ** -0.5, ints(places))
    check_rows(cache, q, out, lse, d ** -0.5, last_tokens(cache, places))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (4, 1), (6, 2), (8, 1), (9, 1), (16, 1), (17, 1), (40, 1), (64, 2), (48, 16)])
@pytest.mark.parametrize("width", [None, 500])
def test_attend_heads(io, hq, hkv, width):
    cache, names = make_cache([5, 300, 64], 16, 16, hkv, 64, io, seed=hq, width=width)
    q = randn((3, hq, 64), io, 2)
    out, lse = attend(cache, q, 0.125, ints(names))
    check_rows(cache, q, out, lse, 0.125, last_tokens(cache, [int(s) for s in names]))


@pytest.mark.parametrize("io,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("window,sink", [(1, 0), (5, 3), (16, 40), (64, 0), (100, 64), (33, 31), (5000, 7), (2 ** 31 - 1, 2 ** 31 - 1), (0, 9)])
def test_attend_window_and_sink(io, d, window, sink):
    cache, names = make_cache([1, 20, 64, 65, 130, 700, 2000], 32, 16, 2, d, io)
    q = randn((7, 4, d), io, 3)
    out, lse = attend(cache, q, d ** -0.5, ints(names), window=window, sink=sink)
    check_rows(cache, q, out, lse, d ** -0.5, last_tokens(cache, [int(s) for s in names]), window, sink)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["token", "head", "gaps", "mixed"])
def test_attend_layouts_layers_and_strided_queries(io, layout):
    cache, names = make_cache([40, 333, 3], 16, 8, 3, 64, io, layers=3, layout=layout)
    q = randn((3, 9, 72), io, 4)[:, ::1, :64]
    for layer in (0, 2):
        out, lse = attend(cache, q, 0.2, ints(names), layer=layer)
        check_rows(cache, q, out, lse, 0.2, last_tokens(cache, [int(s) for s in names]), layer=layer)


def test_attend_pages_status_and_lengths_that_do_not_exist():
    cache, names = make_cache([100, 100, 100, 64], 16, 16, 2, 128)
    a, b, c, d = (int(s) for s in names)
    cache.page_table[a, 1], cache.page_table[a, 3], cache.page_table[b, :] = -1, 10 ** 6, -5
    cache.seq_len[c] = 10 ** 9
    q = randn((4, 8, 128), "bf16", 5)
    out, lse = attend(cache, q, 0.1, ints(names), status=ints([0, 0, 0, 1]))
    length = cache.k.shape[2] * cache.page_table.shape[1]
    cache.seq_len[c] = length                                      # what it is cut to
    for i, p in enumerate(cache.page_table[c].tolist()):
        assert p >= 0 or i >= 7
    held = Held(cache)
    held.length[c] = length
    # the pages of c end at 100 of 112 tokens: the last slots hold NaN, which it sees
    assert np.isnan(f64(out)[2]).all()
    out[2], lse[:, 2] = NAN, NAN
    check_rows(cache, q, out, lse, 0.1, [(0, a, 99), (1, b, 99)], held=held)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_attend_nan_and_infinite_queries_reach_who_sees_them(io):
    import torch
    cache, names = make_cache([100, 100, 100, 100, 100], 16, 16, 2, 64, io)
    row = {i: cache.page_table[int(s)].tolist() for i, s in enumerate(names)}
    k, v = cache.k.view(torch.uint8), cache.v.view(torch.uint8)
    k[0, row[0][1], 3, 0, 7] = 0x7f        # place 0: one key of KV head 0
    v[0, row[1][1], 3, 1, 9] = 0xff        # place 1: one number of V of KV head 1
    k[0, row[2][6], 4:, :, :] = 0x7f       # place 2: behind the last token
    v[0, row[2][6], 4:, :, :] = 0x7f
    q = randn((5, 4, 64), io, 6)
    q[3, 2, 5] = float("nan")
    q[4, 1, 5] = float("inf")
    out, lse = attend(cache, q, 0.125, ints(names))
    o, l = f64(out), f64(lse)
    assert np.isnan(o[0, :2]).all() and np.isnan(l[:2, 0]).all() and np.isfinite(o[0, 2:]).all()
    assert np.isnan(o[1, 2:, 9]).all() and np.isfinite(np.delete(o[1], 9, 1)).all() and np.isfinite(o[1, :2]).all() and np.isfinite(l[:, 1]).all()
    assert np.isfinite(o[2]).all()
    assert np.isnan(o[3, 2]).all() and np.isfinite(np.delete(o[3], 2, 0)).all()
    assert np.isnan(o[4, 1]).all() and np.isfinite(np.delete(o[4], 1, 0)).all()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 32])
@pytest.mark.parametrize("n", [40, 5000])
def test_attend_infinite_keys_and_values(io, d, n):
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
    q = randn((2, 4, d), io, 1)
    q[1, :, 5] = -1.0
    out, lse = attend(cache, q, 0.1, ints(names))
    o = f64(out)
    assert (o[0, :, 3] == np.inf).all() and (o[0, :, 4] == -np.inf).all() and np.isfinite(np.delete(o[0], [3, 4], 1)).all()
    # a score of -inf weighs what -2^127 weighs
    cache.k_scale[0, p, slot // 16] = 245
    o2, l2 = attend(cache, q, 0.1, ints(names))
    assert np.isfinite(o[1]).all() and np.isfinite(f64(lse)[:, 1]).all() and torch.equal(out[1], o2[1]) and torch.equal(lse[:, 1], l2[:, 1])
    cache.k_scale[0, p, slot // 16] = 247
    q[1, :, 5] = 1.0
    out, lse = attend(cache, q, 0.1, ints(names))
    assert np.isnan(f64(out)[1]).all()


def test_attend_many_places_and_one_long_sequence():
    cache, names = make_cache([1 + 37 * i % 900 for i in range(300)] + [40000], 32, 32, 2, 128, extra_seqs=5)
    places = [int(s) for s in names]
    q = randn((301, 8, 128), "bf16", 7)
    out, lse = attend(cache, q, 0.088, ints(places))
    rows = last_tokens(cache, places)
    check_rows(cache, q, out, lse, 0.088, rows)


# ------------------------------------------------------------------------------------------------- append and read
def same_cache(cache, held):
    """Codes, scales and map are the oracle's; NaN may have either sign."""
    import torch
    for got, want in ((cache.k.view(torch.uint8), held.k), (cache.v.view(torch.uint8), held.v)):
        got = got.cpu().numpy()
        diff = (got != want) & ~(((got & 0x7f) == 0x7f) & ((want & 0x7f) == 0x7f))
        assert not diff.any(), f"{diff.sum()} codes differ, the first at {np.argwhere(diff)[0]}: {got[diff][:4]} and {want[diff][:4]}"
    for got, want in ((cache.k_scale, held.ks), (cache.v_scale, held.vs)):
        assert np.array_equal(got.cpu().numpy(), want)
    for got, want in ((cache.page_table, held.table), (cache.seq_len, held.length), (cache.page_ref, held.ref)):
        assert np.array_equal(got.cpu().numpy(), want)


def grow(cache, held, seqs, new, k_new, v_new, layers=(0,)):
    """reserve, and append in some layers, here and in the oracle"""
    import torch
    cu = np.concatenate([[0], np.cumsum(new)])
    status = ints([9] * len(seqs))
    P.dcp_cache_reserve(cache, ints(seqs), status, n_new=ints(new))
    for layer in layers:
        P.dcp_cache_append(cache, k_new, v_new, seqs=ints(seqs), cu_new=ints(cu), status=status, layer=layer)
    torch.cuda.synchronize()
    m = held.map()
    codes = m.reserve(seqs, new)
    assert status.tolist() == codes
    for layer in layers:
        e4m3.append(m, held.ks, held.vs, held.block, seqs, cu, f64(k_new), f64(v_new), codes, layer)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 32])
@pytest.mark.parametrize("page,block,layout", [(1, 1, "token"), (16, 16, "head"), (20, 10, "gaps"), (37, 37, "token"), (64, 8, "mixed"), (64, 1, "gaps"), (256, 256, "token")])
def test_append_and_read(io, d, page, block, layout):
    import torch
    lens, new = [0, 1, 5, 16, 37, 63, 64, 300, 7], [1, 40, 0, 3, 300, 1, 2, 17, 5]
    cache, names = make_cache(lens, page, block, 3, d, io, layers=2, spare=600 // page + 12, width=700 // page + 3, layout=layout, seed=d)
    seqs, held = [int(s) for s in names] + [-1], Held(cache)
    new = new + [0]
    k_new, v_new = randn((sum(new), 3, d), io, 1, 3.0), randn((sum(new), 3, d + 16), io, 2)[:, :, :d]
    k_new[::7] *= 2.0 ** -9      # below the normal codes
    k_new[::5, 1] = 0
    grow(cache, held, seqs, new, k_new, v_new, layers=(1,))
    same_cache(cache, held)
    # back, more tokens than were new, and more than some sequences have
    back = [min(n + 9, held.length[s] + 2) if s >= 0 else 0 for n, s in zip(new, seqs)]
    cu = np.concatenate([[2], 2 + np.cumsum(back)])
    for dtype_out in (k_new.dtype,):
        k_out = torch.full((cu[-1] + 3, 3, d + 16), NAN, dtype=dtype_out, device="cuda")[:, :, :d]
        v_out = torch.full((cu[-1] + 3, 3, d), NAN, dtype=dtype_out, device="cuda")
        P.dcp_cache_read(cache, k_out, v_out, seqs=ints(seqs), cu_new=ints(cu), layer=1)
        torch.cuda.synchronize()
        want_k, want_v = (np.full((cu[-1] + 3, 3, d), NAN) for _ in range(2))
        for i, s in enumerate(seqs):
            if s < 0:
                continue
            pos = np.arange(held.length[s] - back[i], held.length[s])
            rows = cu[i] + np.arange(back[i])
            _, k, v = held.values(s, pos[pos >= 0], 1)
            want_k[rows[pos >= 0]], want_v[rows[pos >= 0]] = k, v
        assert np.array_equal(f64(k_out), want_k, equal_nan=True) and np.array_equal(f64(v_out), want_v, equal_nan=True)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("block", [1, 2, 32])
@pytest.mark.parametrize("tokens", [1025, 17000])
def test_append_of_many_tokens(io, block, tokens):
    """The forms of many tokens, whose workgroups have some or many of them; the last block of a sequence is partly full and begins the next append's."""
    import torch
    page, d, hkv = 64, 32, 3
    cache = P.Cache.empty(1, tokens // 32 + 8, page, hkv, d, 3, tokens // page + 4, torch.float8_e4m3fn, scale_block=block, io_dtype=dtype_of(io))
    held = Held(cache)
    x, y = randn((tokens, hkv, d), io, 1), randn((tokens, hkv, d), io, 2, 5.0)
    grow(cache, held, [2, -1, 0], [tokens - 40, 0, 40], x, y)
    same_cache(cache, held)
    more = tokens // 2
    grow(cache, held, [0, 2], [more, 5], y[: more + 5], x[: more + 5])
    same_cache(cache, held)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_append_every_bf16_number(io):
    """Each alone in its block: the scale of every size, rounding, infinities and NaN."""
    import torch
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(1024, 1, 64)
    x = torch.zeros((1024, 64, 32), dtype=torch.bfloat16)
    x[:, :, 3] = bits[:, 0]
    cache = P.Cache.empty(1, 64, 16, 64, 32, 1, 64, torch.float8_e4m3fn, scale_block=1, io_dtype=dtype_of(io))
    held = Held(cache)
    x = x.to(dtype_of(io)).cuda()
    grow(cache, held, [0], [1024], x, x)
    same_cache(cache, held)
    k, v = torch.empty_like(x), torch.empty_like(x)
    P.dcp_cache_read(cache, k, v, cu_new=ints([0, 1024]))
    want = f64(x)[:, :, 3]
    got = f64(k)[:, :, 3]
    fine = np.isfinite(want)
    assert np.isnan(got[~fine]).all()
    # half a step of 4 significant bits; below 2^-126, the least normal number, half of that
    top = fine & (np.abs(want) < 2.0 ** 128 * (1 - 2.0 ** -5))
    assert (np.abs(got[top] - want[top]) <= np.maximum(2.0 ** -4 * np.abs(want[top]), 2.0 ** -127)).all()
    assert np.isinf(got[fine & ~top]).all()


@pytest.mark.parametrize("block", [4, 16, 64])
def test_append_token_by_token_with_growing_values(block):
    """Every step needs a larger scale for some block, and what it holds already is rounded again."""
    import torch
    cache = P.Cache.empty(1, 12, 64, 2, 64, 3, 4, torch.float8_e4m3fn, scale_block=block)
    held = Held(cache)
    for step in range(70):
        x = randn((2, 2, 64), "bf16", step, 1.3 ** (step % 40))
        grow(cache, held, [2, 0], [1, 1], x, -x)
        if step % 9 == 0 or step == 69:
            same_cache(cache, held)


def test_append_leaves_out_what_has_no_place():
    import torch
    cache, names = make_cache([30, 20, 10], 16, 8, 2, 64, spare=5, width=4)
    held = Held(cache)
    a, b, c = (int(s) for s in names)
    x = randn((40, 2, 64), "bf16", 1)
    # more tokens than the sequence has; a status; a sequence that is none; rows behind n_tokens
    P.dcp_cache_append(cache, x, x, seqs=ints([a, b, 77, c]), cu_new=ints([0, 33, 35, 36, 50]), status=ints([0, 1, 0, 0]))
    torch.cuda.synchronize()
    m = held.map()
    e4m3.append(m, held.ks, held.vs, 8, [a], [0, 33], f64(x), f64(x), [0])
    e4m3.append(m, held.ks, held.vs, 8, [c], [36, 50], np.concatenate([f64(x), np.zeros((20, 2, 64))]), np.concatenate([f64(x), np.zeros((20, 2, 64))]), [0], n_tokens=40)
    same_cache(cache, held)


def test_append_from_a_begin_below_zero_writes_the_tokens_that_are_there():
    import torch
    cache, names = make_cache([25, 40], 16, 16, 2, 64)
    a, before = int(names[0]), Held(cache)
    x, y = randn((3, 2, 64), "bf16", 1), randn((3, 2, 64), "bf16", 2)
    P.dcp_cache_append(cache, x, y, seqs=ints([a]), cu_new=ints([-2, 3]))
    torch.cuda.synchronize()
    after = Held(cache)
    j, k, v = after.values(a, np.arange(25))
    # a code is off by half a step, 2^-4 of it, or 2^-10 units where it is below the normal codes
    for got, want, scales in ((k, x, after.ks), (v, y, after.vs)):
        unit = 2.0 ** (scales[0, after.table[a][1], 0].astype(np.float64) - 127)[None, :, None]
        assert (np.abs(got[22:] - f64(want)) <= np.maximum(2.0 ** -4 * np.abs(f64(want)), 2.0 ** -10 * unit)).all()
    _, k0, v0 = before.values(a, np.arange(22))
    for got, want, scales in ((k, k0, after.ks), (v, v0, after.vs)):
        unit = 2.0 ** (scales[0, after.table[a][1], 0].astype(np.float64) - 127)[None, :, None]
        assert (np.abs(got[:22] - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * unit)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(128, 16), (32, 20)])
def test_read_of_the_other_caches_copies(dtype, d, page):
    import torch
    from tests.test_gpu_paged import make_cache as make_other
    cache, names = make_other([0, 5, 300], page, 2, d, dtype, layers=2)
    table, length = cache.page_table.cpu().numpy(), cache.seq_len.cpu().numpy()
    cu = [0, 2, 6, 206]
    for many in (1, 40):   # up to 1 024 rows and above take another form
        seqs = [int(s) for s in names] * many
        starts = [0] + [206 * i + x for i in range(many) for x in cu[1:]]
        k, v = (torch.full((starts[-1], 2, d), NAN, dtype=dtype_of(dtype), device="cuda") for _ in range(2))
        P.dcp_cache_read(cache, k, v, seqs=ints(seqs), cu_new=ints(starts), layer=1)
        for i, s in enumerate(seqs):
            n = starts[i + 1] - starts[i]
            for y in range(n):
                pos = int(length[s]) - n + y
                want = [torch.full((2, d), NAN)] * 2 if pos < 0 else [x[1, table[s, pos // page], pos % page].float().cpu() for x in (cache.k, cache.v)]
                assert torch.equal(k[starts[i] + y].float().cpu().nan_to_num(7e7), want[0].nan_to_num(7e7)) or i > 4
                if i <= 4:
                    assert torch.equal(v[starts[i] + y].float().cpu().nan_to_num(7e7), want[1].nan_to_num(7e7))
                if i > 4:
                    break
        if many > 1:
            assert torch.equal(k.view(many, 206, 2, d).nan_to_num(7e7), k.view(many, 206, 2, d)[:1].expand(many, -1, -1, -1).nan_to_num(7e7))
            assert torch.equal(v.view(many, 206, 2, d).nan_to_num(7e7), v.view(many, 206, 2, d)[:1].expand(many, -1, -1, -1).nan_to_num(7e7))


# ------------------------------------------------------------------------------------------------- pages that move
@pytest.mark.parametrize("page,block,hkv,d", [(16, 8, 2, 64), (20, 5, 3, 32), (64, 64, 1, 128), (256, 16, 8, 128)])
def test_fork_free_and_compact_take_the_scales_along(page, block, hkv, d):
    import torch
    cache, names = make_cache([3, page, 3 * page + 5, 2 * page - 1, 2 * page + block], page, block, hkv, d, layers=2, spare=9, extra_seqs=5)
    held = Held(cache)
    free = [s for s in range(10) if s not in set(int(x) for x in names)]
    src, dst = [int(s) for s in names[[0, 1, 2, 2]]] + [int(names[4])], free[:5]
    status = ints([9] * 5)
    P.dcp_cache_fork(cache, ints(src), ints(dst), status)
    torch.cuda.synchronize()
    # scales of the page that is being filled go with its tokens
    m = held.map()
    was = held.length.copy()
    assert m.fork(src, dst) == status.tolist() == [0] * 5
    for a, b in zip(src, dst):
        whole, part = divmod(int(was[a]), page)
        if part:
            n = -(-part // block)
            for sc in (held.ks, held.vs):
                sc[:, held.table[b, whole], :n] = sc[:, held.table[a, whole], :n]
    same_cache(cache, held)
    P.dcp_cache_free(cache, ints([src[2], dst[0]]))
    m.free([src[2], dst[0]])
    counts, ws = ints([0, 0]), torch.empty(P.dcp_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    before = held.ref.copy()
    P.dcp_cache_compact(cache, counts, ws)
    torch.cuda.synchronize()
    used = int((before > 0).sum())
    holes, high = [p for p in range(used) if before[p] == 0], [p for p in range(used, len(before)) if before[p] > 0]
    for p, to in zip(high, holes):
        for sc in (held.ks, held.vs):
            sc[:, to] = sc[:, p]
    assert counts.tolist() == m.compact()
    same_cache(cache, held)


@pytest.mark.parametrize("page,block,io", [(8, 4, "bf16"), (5, 1, "f32"), (12, 12, "bf16")])
def test_a_random_life_of_a_cache(page, block, io):
    """Steps in any order, refused ones among them: codes, scales and map against the oracle's after each."""
    import torch
    rng = np.random.default_rng(page)
    layers, hkv, d, n_pages = 2, 2, 32, 40
    cache = P.Cache.empty(layers, n_pages, page, hkv, d, 8, 9, torch.float8_e4m3fn, scale_block=block, io_dtype=dtype_of(io))
    cache.k.view(torch.uint8).fill_(0x7f)
    cache.v.view(torch.uint8).fill_(0x7f)
    held = Held(cache)
    for step in range(60):
        kind = rng.integers(0, 6)
        m = held.map()
        if kind <= 2:
            seqs = [int(x) for x in rng.permutation(9)[:4] - 1]
            new = [int(x) for x in rng.integers(0, 2 * page, 4)]
            k, v = (randn((sum(new), hkv, d), io, 3 * step + x, float(rng.choice([0.01, 1, 30]))) for x in (0, 1))
            grow(cache, held, seqs, new, k, v, layers=range(layers))
        elif kind == 3:
            src, dst = [int(x) for x in rng.integers(-1, 8, 3)], [int(x) for x in rng.integers(0, 8, 3)]
            status, was = ints([9] * 3), held.length.copy()
            P.dcp_cache_fork(cache, ints(src), ints(dst), status)
            codes = m.fork(src, dst)
            assert status.tolist() == codes
            for a, b, code in zip(src, dst, codes):
                if a >= 0 and code == 0 and was[a] % page:
                    n = -(-(int(was[a]) % page) // block)
                    for sc in (held.ks, held.vs):
                        sc[:, held.table[b, was[a] // page], :n] = sc[:, held.table[a, was[a] // page], :n]
        elif kind == 4:
            seqs = [int(x) for x in rng.integers(-1, 8, 2)]
            P.dcp_cache_free(cache, ints(seqs))
            m.free(seqs)
        else:
            counts, ws = ints([0, 0]), torch.empty(P.dcp_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
            P.dcp_cache_compact(cache, counts, ws)
            used = int((held.ref > 0).sum())
            moves = list(zip([p for p in range(used, n_pages) if held.ref[p] > 0], [p for p in range(used) if held.ref[p] == 0]))
            for p, to in moves:
                for sc in (held.ks, held.vs):
                    sc[:, to] = sc[:, p]
            assert counts.tolist() == m.compact()
        torch.cuda.synchronize()
        # entries of the table behind the pages that a sequence holds may be anything
        got = cache.page_table.cpu().numpy()
        for s in range(8):
            held.table[s, m.held(s):] = got[s, m.held(s):]
        same_cache(cache, held)
        live = [s for s in range(8) if held.length[s]]
        if live and step % 3 == 0:
            q = randn((len(live), 4, d), io, step)
            out, lse = attend(cache, q, 0.2, ints(live))
            check_rows(cache, q, out, lse, 0.2, last_tokens(cache, live), held=held)


def test_offsets_past_32_bits():
    """A cache of 6 GiB of keys and as many of values, whose sequences lie at its end."""
    import torch
    layers, pages, page, hkv, d = 3, 16384, 128, 8, 128
    k, v = (torch.zeros((layers, pages, page, hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((layers, pages, 8, hkv), 120, dtype=torch.uint8, device="cuda") for _ in range(2))
    table, length = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), ints([200, 0])
    table[0, :2] = ints([pages - 1, pages - 3])
    ref = torch.ones(pages, dtype=torch.int32, device="cuda")
    ref[pages - 2] = 0
    cache = P.Cache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ref, table, length, k_scale=ks, v_scale=vs)
    x = randn((200, hkv, d), "bf16", 1)
    P.dcp_cache_append(cache, x, x.flip(0).contiguous(), seqs=ints([0]), cu_new=ints([0, 200]), layer=2)
    back = [torch.empty_like(x) for _ in range(2)]
    P.dcp_cache_read(cache, *back, cu_new=ints([0, 200]), layer=2)
    q = randn((1, 16, d), "bf16", 2)
    out, lse = attend(cache, q, 0.1, ints([0]), layer=2)
    held_k, held_v = f64(back[0]), f64(back[1])
    assert (np.abs(held_k - f64(x)) <= np.maximum(2.0 ** -4 * np.abs(f64(x)), 2.0 ** -10 * 2.0 ** -6)).all()   # the scale is at most 2^-6 (4.8 sigma)
    from oracle import paged as OP
    ref_o, ref_l, mean, _ = OP.attend(f64(q)[0], held_k, held_v, 0.1)
    assert (np.abs(f64(out)[0] - ref_o) <= 2.0 ** -8 * np.abs(ref_o) + 2.0 ** -13 * mean).all()
    assert int(k[0].max()) == 0 and int(k[1].max()) == 0 and int(v[2, :-3].max()) == 0
