"""The paged key-value cache and the attention of one new token over it against the 64-bit oracle.

Slots that hold no token, and pages that nobody holds, are filled with NaN: whatever reads one shows it."""
import numpy as np
import pytest

import paper_2510_10620_amd as P
from oracle import paged as OP

pytestmark = pytest.mark.gpu

NAN = float("nan")


def _dtype(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _f64(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


def make_cache(lens, page, hkv, d, dtype="bf16", layers=1, spare=3, extra_seqs=1, width=None, seed=0, layout="token", scale=1.0):
    """A cache whose sequences lie on pages in any order.  layout: "token" [.., page, hkv, d], "head" [.., hkv, page, d], "gaps" (rows
    with room between them).  -> (Cache, sequences of `lens`)"""
    import torch
    rng = np.random.default_rng(seed)
    used = [-(-n // page) for n in lens]
    n_pages, n_seqs = sum(used) + spare, len(lens) + extra_seqs
    width = width or max(1, max(used))
    where, names = rng.permutation(n_pages), rng.permutation(n_seqs)[:len(lens)]
    table, ref, length = np.full((n_seqs, width), -1, np.int32), np.zeros(n_pages, np.int32), np.zeros(n_seqs, np.int32)
    kv = []
    for _ in range(2):
        x = torch.full((layers, n_pages, page, hkv, d), NAN, dtype=torch.float32)
        at = 0
        for s, n in enumerate(lens):
            for p in where[at: at + used[s]]:
                m = min(page, n)
                x[:, p, :m] = torch.from_numpy(rng.standard_normal((layers, m, hkv, d)).astype(np.float32)) * scale
                n -= m
            at += used[s]
        x = x.to(_dtype(dtype))
        if layout == "head":
            y = torch.empty((layers, n_pages, hkv, page, d), dtype=x.dtype, device="cuda").transpose(2, 3)
        elif layout == "gaps":
            y = torch.full((layers, n_pages, page, hkv + 1, d + 8), NAN, dtype=x.dtype, device="cuda")[:, :, :, :hkv, :d]
        else:
            y = torch.empty(x.shape, dtype=x.dtype, device="cuda")
        kv.append(y.copy_(x))
    at = 0
    for s, n in enumerate(lens):
        table[names[s], : used[s]] = where[at: at + used[s]]
        length[names[s]] = n
        at += used[s]
    ref[where[:at]] = 1
    ints = [torch.from_numpy(a).cuda() for a in (ref, table, length)]
    return P.Cache(kv[0], kv[1], *ints), names


def ints(x):
    import torch
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def attend(cache, q, scale, seqs=None, window=0, sink=0, layer=0):
    import torch
    out, lse = torch.full_like(q, NAN), torch.full((q.shape[1], q.shape[0]), NAN, dtype=torch.float32, device="cuda")
    ws = torch.empty(P.dcp_paged_attn_workspace_bytes(cache, q.shape[0], q.shape[1]), dtype=torch.uint8, device="cuda").random_()
    P.dcp_paged_attn_fwd(cache, q, out, lse, scale, ws, seqs=seqs, window=window, sink=sink, layer=layer)
    torch.cuda.synchronize()
    return out, lse


def check(cache, q, out, lse, scale, places, window=0, sink=0, layer=0):
    """Every place of the batch against the oracle.

    With u the half step of fp32 (2^-24), r that of the outputs' type, L keys of D dimensions: a score is off by at most
    (D + 4) u scale sum|q k| (the products and their sum, the scale, and log2 e in it), the exponential by 4 u more, so a weight by
    e = 2 ((D + 4) u size + 4 u) of itself (its own score and the maximum's); the sums by L u; bf16 weights are held in two parts, to 2^-15.
    The output is a quotient of two such sums over |v| and is rounded once."""
    bf16 = cache.k.element_size() == 2
    u, r, d = 2.0 ** -24, 2.0 ** -8 if bf16 else 2.0 ** -24, cache.k.shape[4]
    table, length, page = cache.page_table.cpu().numpy(), cache.seq_len.cpu().numpy(), cache.k.shape[2]
    o, l, qq = _f64(out), _f64(lse), _f64(q)
    worst = 0.0
    for i, s in enumerate(places):
        if s < 0 or s >= len(length):
            assert np.isnan(o[i]).all() and np.isnan(l[:, i]).all(), f"place {i} is padding and was written"
            continue
        j = OP.seen_keys(int(length[s]), window, sink)
        pages = table[s][j // page]
        j, pages = j[(pages >= 0) & (pages < cache.k.shape[1])], pages[(pages >= 0) & (pages < cache.k.shape[1])]
        at = (np.full(len(j), layer), pages, j % page)
        k, v = (_f64(x[tuple(np_index(a) for a in at)]) for x in (cache.k, cache.v))
        ref, ref_l, mean, size = OP.attend(qq[i], k, v, scale)
        if not len(j):
            assert (o[i] == 0).all() and (l[:, i] == -np.inf).all()
            continue
        e = 2 * ((d + 4) * u * size + 4 * u) + 2 * len(j) * u + (2.0 ** -15 if bf16 else 0)
        bound = r * np.abs(ref) + 1.01 * (2 * e[:, None] * mean)
        bad = np.abs(o[i] - ref) / bound
        assert bad.max() <= 1, f"place {i} (sequence {s}, {len(j)} keys): out is {bad.max():.2f} times its bound off"
        bad_l = np.abs(l[:, i] - ref_l) / (e + 2 * u * np.abs(ref_l) + 4 * u)
        assert bad_l.max() <= 1, f"place {i} (sequence {s}, {len(j)} keys): LSE is {bad_l.max():.2f} times its bound off"
        worst = max(worst, bad.max(), bad_l.max())
    return worst


def np_index(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int64)).cuda()


def randn(shape, dtype, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(_dtype(dtype)).cuda()


EDGES = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 400, 1000]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 32])
@pytest.mark.parametrize("page", [1, 8, 16, 20, 37, 64])
def test_lengths_and_pages(dtype, d, page):
    cache, names = make_cache(EDGES, page, 2, d, dtype, seed=page)
    places = [int(s) for s in names] + [-1]
    q = randn((len(places), 8, d), dtype, 1)
    out, lse = attend(cache, q, d ** -0.5, ints(places))
    check(cache, q, out, lse, d ** -0.5, places)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (2, 1), (4, 1), (6, 2), (7, 1), (8, 1), (9, 1), (16, 1), (17, 1), (40, 1), (64, 2), (48, 16)])
@pytest.mark.parametrize("width", [None, 500])
def test_heads(dtype, hq, hkv, width):
    """width 500: a table with room for long sequences, whose items may be cut."""
    cache, names = make_cache([5, 300, 64], 16, hkv, 64, dtype, seed=hq, width=width)
    q = randn((3, hq, 64), dtype, 2)
    out, lse = attend(cache, q, 0.125, ints(names))
    check(cache, q, out, lse, 0.125, [int(s) for s in names])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (5, 3), (16, 40), (64, 0), (100, 64), (33, 31), (5000, 7), (2 ** 31 - 1, 2 ** 31 - 1), (0, 9)])
def test_window_and_sink(dtype, d, window, sink):
    cache, names = make_cache([0, 1, 40, 64, 97, 128, 300, 1111], 24, 2, d, dtype, seed=3)
    places = [int(s) for s in names]
    q = randn((len(places), 4, d), dtype, 4)
    out, lse = attend(cache, q, d ** -0.5, ints(places), window, sink)
    check(cache, q, out, lse, d ** -0.5, places, window, sink)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["token", "head", "gaps"])
def test_layouts_layers_and_strided_queries(dtype, layout):
    import torch
    cache, names = make_cache([70, 1, 333], 32, 3, 64, dtype, layers=3, seed=5, layout=layout)
    places = [-1, int(names[2]), 4000, int(names[0]), int(names[2]), -7, int(names[1])]      # a sequence twice, padding, no sequence
    big = torch.full((len(places), 9, 80), NAN, dtype=_dtype(dtype), device="cuda")
    q = big[:, 1:7, 8:72].copy_(randn((len(places), 6, 64), dtype, 6))
    for layer in (0, 2):
        out, lse = attend(cache, q, 0.2, ints(places), layer=layer)
        check(cache, q, out, lse, 0.2, places, layer=layer)
    wide = torch.full((len(places), 8, 72), NAN, dtype=_dtype(dtype), device="cuda")
    lse2, ws = torch.empty_like(lse), torch.empty(P.dcp_paged_attn_workspace_bytes(cache, len(places), 6), dtype=torch.uint8, device="cuda")
    P.dcp_paged_attn_fwd(cache, q, wide[:, :6, :64], lse2, 0.2, ws, seqs=ints(places), layer=2)
    assert torch.equal(torch.nan_to_num(wide[:, :6, :64]), torch.nan_to_num(out))
    assert torch.isnan(wide[:, 6:]).all() and torch.isnan(wide[:, :, 64:]).all()


def test_without_seqs_place_i_is_sequence_i():
    cache, names = make_cache([70, 1, 333, 50], 32, 1, 128, extra_seqs=0, seed=8)
    q = randn((3, 4, 128), "bf16", 6)
    out, lse = attend(cache, q, 0.1)
    check(cache, q, out, lse, 0.1, [0, 1, 2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_far_away_maxima(dtype):
    """Scores of hundreds, the largest at either end or in the middle."""
    cache, names = make_cache([2000, 2000, 2000], 16, 1, 64, dtype, seed=9)
    for s, at in zip(names, (0, 999, 1999)):
        cache.k[0, cache.page_table[s, at // 16].item(), at % 16] *= 30
    q = randn((3, 4, 64), dtype, 10) * 4
    out, lse = attend(cache, q, 0.5, ints(names))
    check(cache, q, out, lse, 0.5, [int(s) for s in names])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 32), ("f32", 64)])
def test_pages_and_lengths_that_do_not_exist(dtype, d):
    """Entries that name no page hold nothing, lengths are cut to the table's row: nothing out of range is read."""
    import torch
    cache, names = make_cache([100, 200, 300, 77], 16, 2, d, dtype, seed=11)
    a, b, c, e = (int(s) for s in names)
    cache.page_table[a, 2], cache.page_table[a, 5] = -1, 1 << 30
    cache.page_table[b, :13] = cache.k.shape[1]
    cache.page_table[c, 0] = -(1 << 31)
    width = cache.page_table.shape[1]
    cache.seq_len[e] = -5
    q = randn((4, 4, d), dtype, 12)
    out, lse = attend(cache, q, 0.1, ints(names))
    cache.seq_len[e] = 0
    check(cache, q, out, lse, 0.1, [a, b, c, e])
    full = cache.page_table[c].clone()
    cache.seq_len[c] = 1 << 30                          # as if the row were full
    cache.k[torch.isnan(cache.k)] = 0.5
    cache.v[torch.isnan(cache.v)] = 0.5
    out, lse = attend(cache, q[2:3].contiguous(), 0.1, ints([c]))
    cache.seq_len[c] = width * 16
    assert torch.equal(full, cache.page_table[c])
    check(cache, q[2:3], out, lse, 0.1, [c])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_inf_and_nan_reach_who_sees_them(dtype, d):
    import torch
    cache, names = make_cache([90, 300, 500, 40], 16, 2, d, dtype, seed=13)
    a, b, c, e = (int(s) for s in names)

    def at(s, j):
        return 0, int(cache.page_table[s, j // 16]), j % 16

    q = randn((4, 4, d), dtype, 14)
    clean, clean_l = attend(cache, q, 0.1, ints(names), 64, 8)
    cache.v[at(b, 200)][:] = float("inf")               # outside the window: unseen
    cache.k[at(b, 100)][:] = NAN
    cache.k[at(c, 480)][0, :] = NAN                     # seen, KV head 0
    cache.v[at(a, 3)][1, 5] = float("inf")              # seen through the sink, KV head 1, one column
    cache.v[at(e, 39)][0, 7] = -float("inf")
    out, lse = attend(cache, q, 0.1, ints(names), 64, 8)
    same = torch.ones_like(out, dtype=torch.bool)
    same[2, :2] = False
    same[0, 2:, 5] = False
    same[3, :2, 7] = False
    assert torch.equal(out[same], clean[same])
    assert torch.isnan(out[2, :2]).all() and torch.isnan(lse[:2, 2]).all()
    assert (out[0, 2:, 5] == float("inf")).all() and (out[3, :2, 7] == -float("inf")).all()
    lse[:2, 2] = clean_l[:2, 2]
    assert torch.equal(lse, clean_l)
    # keys whose scores are all -inf weigh nothing
    cache.k[at(e, 39)][0, :] = 0
    for j in range(40):
        cache.k[at(e, j)][1, 0] = -float("inf")
    q2 = q.clone()
    q2[3, 2:, 0] = 1.0
    out, lse = attend(cache, q2, 0.1, ints(names))
    assert (out[3, 2:] == 0).all() and (lse[2:, 3] == -float("inf")).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 32), ("f32", 64)])
@pytest.mark.parametrize("n", [1, 3, 64, 150, 600])
def test_short_sequences_taken_whole_or_cut(dtype, d, n):
    """Up to 90 tokens in a table without room for more (a workgroup an item, or several items one after the other), and in one with."""
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, 91, n)]
    lens[0] = 90
    for width in (None, 300):
        cache, names = make_cache(lens, 16, 4, d, dtype, seed=n, width=width)
        places = [int(s) for s in names] + [-1]
        q = randn((len(places), 8, d), dtype, 70)
        out, lse = attend(cache, q, d ** -0.5, ints(places))
        check(cache, q, out, lse, d ** -0.5, places)
        out, lse = attend(cache, q, d ** -0.5, ints(places), 20, 3)
        check(cache, q, out, lse, d ** -0.5, places, 20, 3)


def test_many_places_and_one_long_sequence():
    rng = np.random.default_rng(15)
    lens = [int(x) for x in rng.integers(0, 200, 400)] + [30000, 1]
    cache, names = make_cache(lens, 16, 1, 64, seed=16)
    places = [int(s) for s in names]
    q = randn((len(places), 4, 64), "bf16", 17)
    out, lse = attend(cache, q, 0.125, ints(places))
    check(cache, q, out, lse, 0.125, places)
    out, lse = attend(cache, q[-2:].contiguous(), 0.125, ints(places[-2:]))
    check(cache, q[-2:], out, lse, 0.125, places[-2:])


def test_thousands_of_places():
    """More places than a workgroup has threads: twenty a thread."""
    rng = np.random.default_rng(72)
    lens = [int(x) for x in rng.integers(0, 70, 60)]
    cache, names = make_cache(lens, 16, 2, 32, seed=73, width=100)
    places = [int(s) for s in rng.choice(names, 5000)]
    places[0] = places[17] = places[4999] = -1
    q = randn((5000, 4, 32), "bf16", 74)
    out, lse = attend(cache, q, 0.2, ints(places))
    check(cache, q, out, lse, 0.2, places)


@pytest.mark.parametrize("dtype,hq,hkv", [("bf16", 4, 1), ("f32", 2, 2)])
def test_long_sequences_few_heads(dtype, hq, hkv):
    cache, names = make_cache([20011, 9000, 31], 64, hkv, 128, dtype, seed=18)
    q = randn((3, hq, 128), dtype, 19)
    out, lse = attend(cache, q, 128 ** -0.5, ints(names))
    check(cache, q, out, lse, 128 ** -0.5, [int(s) for s in names])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    """Pages whose first byte lies beyond 2^32 of either tensor, in the second layer."""
    import torch
    page, hkv, d = 64, 8, 128
    per_page = page * hkv * d * (2 if dtype == "bf16" else 4)
    n_pages = (1 << 32) // per_page // 2 + 20
    k, v = (torch.zeros((2, n_pages, page, hkv, d), dtype=_dtype(dtype), device="cuda") for _ in range(2))
    table = torch.tensor([[n_pages - 1, 3, n_pages - 7], [n_pages - 2, n_pages - 3, 0]], dtype=torch.int32, device="cuda")
    ref = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    ref[table.flatten().long()] = 1
    cache = P.Cache(k, v, ref, table, ints([150, 0]))
    new = randn((192, hkv, d), dtype, 20), randn((192, hkv, d), dtype, 21)
    P.dcp_cache_free(cache, ints([1]))
    cache.page_table[1] = table[1]
    status = ints([9])
    cache.seq_len[1] = 130
    ref[table[1].long()] = 1
    cu = ints([0, 130])
    P.dcp_cache_append(cache, new[0][:130], new[1][:130], seqs=ints([1]), cu_new=cu, layer=1)
    for t, x in ((k, new[0]), (v, new[1])):
        got = t[1][table[1].clone().long().clamp(min=0)].flatten(0, 1)
        assert torch.equal(got[:128], x[:128])
    for j in (0, 2):
        k[1, table[0, j].item()] = new[0][64 * j: 64 * j + 64]
        v[1, table[0, j].item()] = new[1][64 * j: 64 * j + 64]
    q = randn((2, 16, d), dtype, 22)
    out, lse = attend(cache, q, d ** -0.5, ints([0, 1]), layer=1)
    check(cache, q, out, lse, d ** -0.5, [0, 1], layer=1)
    assert status.item() == 9


# ------------------------------------------------------------------------------------------------ the map
def mirror(cache):
    """The oracle's map of a cache: contents as raw words, so that NaN compare."""
    import torch
    words = torch.int16 if cache.k.element_size() == 2 else torch.int32
    return OP.PagedMap(cache.k.shape[2], cache.page_ref.cpu().numpy().copy(), cache.page_table.cpu().numpy().copy(), cache.seq_len.cpu().numpy().copy(),
                       *(x.contiguous().view(words).cpu().numpy().copy() for x in (cache.k, cache.v)))


def same_map(cache, m):
    got = mirror(cache)
    for name in ("ref", "length", "table", "k", "v"):
        assert np.array_equal(getattr(got, name), getattr(m, name)), name


def words(x):
    import torch
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32).cpu().numpy()


def reserve(cache, m, seqs, new):
    import torch
    status = ints([7] * len(seqs))
    P.dcp_cache_reserve(cache, ints(seqs), status, n_new=ints(new))
    torch.cuda.synchronize()
    want = m.reserve(seqs, new)
    assert status.tolist() == want
    return status


def append(cache, m, seqs, new, status, layer, seed):
    import torch
    dtype = "bf16" if cache.k.element_size() == 2 else "f32"
    cu = np.concatenate([[0], np.cumsum(new)])
    k, v = (randn((int(cu[-1]), *cache.k.shape[3:]), dtype, seed + x) for x in (0, 1))
    P.dcp_cache_append(cache, k, v, seqs=ints(seqs), cu_new=ints(cu), status=status, layer=layer)
    torch.cuda.synchronize()
    m.append(seqs, cu, words(k), words(v), status.tolist(), layer)


@pytest.mark.parametrize("dtype,page,layout", [("bf16", 16, "token"), ("f32", 5, "token"), ("bf16", 1, "gaps"), ("bf16", 64, "head"), ("f32", 8, "gaps")])
def test_a_random_life_of_a_cache(dtype, page, layout):
    """Sequences that grow, fork, end and are compacted, in any order, until pages run out, against the oracle."""
    import torch
    rng = np.random.default_rng(page)
    lens = [0, 3, 2 * page, 5 * page + 1, page, 0, 40]
    cache, _ = make_cache(lens, page, 2, 32, dtype, layers=2, spare=25, extra_seqs=6, width=45, seed=page, layout=layout)
    m = mirror(cache)
    n_seqs = len(m.length)
    ws = torch.empty(P.dcp_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda").random_()
    seen = set()
    for step in range(60):
        n = int(rng.integers(1, 9))
        do = rng.choice(["grow", "grow", "grow", "fork", "free", "compact"])
        if do == "grow":
            seqs = [int(s) for s in rng.integers(-2, n_seqs + 2, n)]
            new = [int(x) for x in rng.integers(-1, 3 * page + 2, n)]
            status = reserve(cache, m, seqs, new)
            seen.update(status.tolist())
            new = [max(0, x) for x in new]
            for layer in range(2):
                append(cache, m, seqs, new, status, layer, 1000 * step + layer)
        elif do == "fork":
            src, dst = ([int(s) for s in rng.integers(-1, n_seqs + 1, n)] for _ in range(2))
            if rng.random() < 0.5:   # mostly empty targets
                empty = np.flatnonzero(m.length == 0)
                dst = [int(x) for x in rng.permutation(empty)[:n]] + dst[len(empty):]
                dst = (dst + src)[:n]
            status = ints([7] * n)
            P.dcp_cache_fork(cache, ints(src), ints(dst), status)
            torch.cuda.synchronize()
            want = m.fork(src, dst)
            assert status.tolist() == want
            seen.update(want)
        elif do == "free":
            seqs = [int(s) for s in rng.integers(-2, n_seqs + 2, min(n, 3))]
            P.dcp_cache_free(cache, ints(seqs + seqs[:1]))
            torch.cuda.synchronize()
            m.free(seqs)
        else:
            counts = ints([-1, -1])
            P.dcp_cache_compact(cache, counts, ws)
            torch.cuda.synchronize()
            assert counts.tolist() == m.compact()
        same_map(cache, m)
    assert seen == {OP.OK, OP.FULL, OP.BAD}


@pytest.mark.parametrize("n_pages,taken", [(1, 0), (63, 5), (8192, 8000), (8193, 4000), (70001, 69990), (70001, 3)])
def test_free_pages_anywhere_in_a_large_map(n_pages, taken):
    """Few free pages among many, or many; the last page; a call that takes all, then one that finds none, then all given back."""
    import torch
    rng = np.random.default_rng(n_pages + taken)
    held = rng.permutation(n_pages)[:taken]
    n_seqs, width = 6, n_pages
    ref, table, length = np.zeros(n_pages, np.int32), np.full((n_seqs, width), -1, np.int32), np.zeros(n_seqs, np.int32)
    ref[held] = 1
    table[5, :taken], length[5] = held, taken
    kv = [torch.zeros((1, n_pages, 1, 1, 32), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = P.Cache(*kv, *(torch.from_numpy(x).cuda() for x in (ref, table, length)))
    m = mirror(cache)
    free = n_pages - taken
    reserve(cache, m, [0, 1, 2, 3], [free // 3, 0, free - free // 3, 0])
    same_map(cache, m)
    reserve(cache, m, [3, 1, 4], [0, 1, 0])
    same_map(cache, m)
    P.dcp_cache_free(cache, ints([5, 0]))
    m.free([5, 0])
    same_map(cache, m)
    # the third place finds some pages, not enough: it gives them back; the fourth needs one and is behind it
    left = n_pages - int((m.ref > 0).sum())
    st = reserve(cache, m, [3, 0, 4, 1], [left // 2, left // 4, left, 1])
    assert left == 0 or st.tolist()[2:] == [OP.FULL, OP.FULL]
    same_map(cache, m)
    counts, ws = ints([0, 0]), torch.empty(P.dcp_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda").random_()
    P.dcp_cache_compact(cache, counts, ws)
    torch.cuda.synchronize()
    assert counts.tolist() == m.compact()
    same_map(cache, m)


def test_many_places_in_one_call():
    """The most places and sequences: sums over several rounds, a sequence named twice."""
    import torch
    n = P.DCP_CACHE_MAX_SEQS
    rng = np.random.default_rng(23)
    kv = [torch.zeros((1, 20000, 4, 1, 32), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = P.Cache.empty(1, 20000, 4, 1, 32, n, 8, torch.bfloat16)
    cache = P.Cache(*kv, cache.page_ref, cache.page_table, cache.seq_len)
    m = mirror(cache)
    seqs = [int(s) for s in rng.permutation(n)]
    seqs[100], seqs[9000] = seqs[9000], seqs[101]
    new = [int(x) for x in rng.integers(0, 9, n)]
    st = ints([7] * n)
    P.dcp_cache_reserve(cache, ints(seqs), st, n_new=ints(new))
    # the oracle's search for free pages is slow: a plain count of the same rule
    want, page, named, full = [], 0, set(), False
    for s, x in zip(seqs, new):
        need = -(-x // 4)
        if s in named:
            want.append(OP.BAD)
            continue
        named.add(s)
        if need and (full or page + need > 20000):
            full = True
            want.append(OP.FULL)
            continue
        m.table[s, :need] = np.arange(page, page + need)
        m.ref[page: page + need] = 1
        m.length[s] = x
        page += need
        want.append(OP.OK)
    assert st.tolist() == want
    same_map(cache, m)
    P.dcp_cache_free(cache, ints(range(n)))
    m.free(range(n))
    same_map(cache, m)


def test_append_leaves_out_what_has_no_place():
    """Tokens before the first place, behind the last and beyond the array, places without room, one token per place."""
    import torch
    cache, names = make_cache([20, 6, 40, 3], 8, 2, 64, layers=1, extra_seqs=0, seed=24)
    m = mirror(cache)
    a, b, c, e = (int(s) for s in names)
    k, v = randn((30, 2, 64), "bf16", 25), randn((30, 2, 64), "bf16", 26)
    # rows 0 and 1 belong to nobody; place 1 has more tokens than its sequence: its first are left out; place 3 reaches beyond the array
    cu = [2, 7, 16, 16, 40]
    P.dcp_cache_append(cache, k, v, seqs=ints([a, b, e, c]), cu_new=ints(cu))
    for s, lo, hi in ((a, 2, 7), (b, 7, 16), (c, 16, 40)):
        for t in range(lo, min(hi, 30)):
            pos = int(m.length[s]) - (hi - t)
            if pos >= 0:
                m.k[0, m.table[s, pos // 8], pos % 8], m.v[0, m.table[s, pos // 8], pos % 8] = words(k)[t], words(v)[t]
    torch.cuda.synchronize()
    same_map(cache, m)
    P.dcp_cache_append(cache, k[:5], v[:5], seqs=ints([e, -1, 99, a, c]), status=ints([0, 0, 0, 1, 0]))
    for s, t in ((e, 0), (c, 4)):
        pos = int(m.length[s]) - 1
        m.k[0, m.table[s, pos // 8], pos % 8], m.v[0, m.table[s, pos // 8], pos % 8] = words(k)[t], words(v)[t]
    torch.cuda.synchronize()
    same_map(cache, m)
    big = torch.full((3, 3, 72), NAN, dtype=torch.bfloat16, device="cuda")
    big[:, 1:, :64] = k[5:8]
    P.dcp_cache_append(cache, big[:, 1:, :64], v[5:8], seqs=ints([a, b, c]))
    for s, t in ((a, 5), (b, 6), (c, 7)):
        pos = int(m.length[s]) - 1
        m.k[0, m.table[s, pos // 8], pos % 8], m.v[0, m.table[s, pos // 8], pos % 8] = words(k)[t], words(v)[t]
    torch.cuda.synchronize()
    same_map(cache, m)


def test_maps_with_pages_that_do_not_exist():
    """Nothing follows a page number or a length out of range."""
    import torch
    cache, names = make_cache([30, 20, 25], 8, 1, 32, spare=4, width=6, seed=27)
    a, b, c = (int(s) for s in names)
    cache.page_table[a, 1], cache.page_table[a, 3] = 1 << 20, -9
    free_seq = [s for s in range(4) if s not in (a, b, c)][0]
    k0, v0 = cache.k.clone(), cache.v.clone()
    st = ints([7])
    P.dcp_cache_fork(cache, ints([a]), ints([free_seq]), st)
    assert st.item() == OP.OK and cache.seq_len[free_seq].item() == 30
    assert torch.equal(torch.nan_to_num(cache.k), torch.nan_to_num(k0)) and torch.equal(torch.nan_to_num(cache.v), torch.nan_to_num(v0))
    P.dcp_cache_append(cache, randn((30, 1, 32), "bf16", 28), randn((30, 1, 32), "bf16", 29), seqs=ints([a]), cu_new=ints([0, 30]))
    P.dcp_cache_free(cache, ints([a, free_seq]))
    assert cache.page_ref.min().item() == 0 and cache.page_ref.sum().item() == 3 + 4 + 2   # the two whose entries are lost stay held
    cache.seq_len[b] = 1 << 30
    P.dcp_cache_reserve(cache, ints([b]), st)
    assert st.item() == OP.BAD                          # no room left in the row
    counts, ws = ints([0, 0]), torch.empty(P.dcp_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    P.dcp_cache_compact(cache, counts, ws)
    assert counts.tolist()[0] == 9


# ------------------------------------------------------------------------------------------------ together
def _prefill_then_decode(dtype, d, graph, window=0, sink=0, block=32):
    """A prompt's keys and values go into the pages, dcp_block_attn_fwd reads them there as block buffers, then tokens are decoded: room,
    keys and values, attention.  Everything against the oracle over the tokens themselves."""
    import torch
    rng = np.random.default_rng(30)
    hq, hkv, page, layers, scale = 4, 2, block, 2, d ** -0.5
    prompts, steps = [70, 1, 33, 128], 7
    cache = P.Cache.empty(layers, 30, page, hkv, d, 6, 10, _dtype(dtype))
    cache.k.fill_(NAN)
    cache.v.fill_(NAN)
    rows = [4, 0, 5, 2]
    seqs = ints(rows + [-1])
    cu = np.concatenate([[0], np.cumsum(prompts)]).astype(np.int32)
    T = int(cu[-1])
    status = ints([7] * 5)
    P.dcp_cache_reserve(cache, seqs, status, n_new=ints(prompts + [0]))
    assert status.tolist() == [0] * 5
    K = [[randn((T + steps * 5, hkv, d), dtype, 31 + 2 * layer + x) for x in (0, 1)] for layer in range(layers)]
    for layer in range(layers):
        P.dcp_cache_append(cache, K[layer][0][:T], K[layer][1][:T], seqs=seqs, cu_new=ints(list(cu) + [T]), status=status, layer=layer)
    # prefill of layer 1 from the pages: kv_slot is the page of every block
    if window:
        table = P.dcp_build_block_table_window(cu, block, window, sink)
    else:
        from paper_2510_10620_amd import workloads as W
        table = P.dcp_build_block_table(cu, block, W.attn_ranges(W.MaskSpec("causal"), cu))
    plan = P.dcp_plan_create(cu, block, table)
    if window:
        P.dcp_plan_set_window(plan, window, sink)
    pages = cache.page_table.cpu().numpy()
    kv_slot = [int(p) for s, n in zip(rows, prompts) for p in pages[s][: -(-n // page)]]
    P.dcp_plan_set_block_buffers(plan, np.arange(len(kv_slot)), len(kv_slot), kv_slot, 30)
    start, length = plan.export("BLK_START"), plan.export("BLK_LEN")
    q = randn((T, hq, d), dtype, 40)
    qb, ob = torch.zeros((len(kv_slot) * page, hq, d), dtype=q.dtype, device="cuda"), torch.zeros((len(kv_slot) * page, hq, d), dtype=q.dtype, device="cuda")
    lb = torch.zeros((hq, len(kv_slot) * page), dtype=torch.float32, device="cuda")
    for b, (s0, n) in enumerate(zip(start, length)):
        qb[b * page: b * page + n] = q[s0: s0 + n]
    P.dcp_block_attn_fwd(plan, qb, cache.k[1].flatten(0, 1), cache.v[1].flatten(0, 1), ob, lb, scale)
    # the last token of every prompt, once more through the pages
    last = [int(cu[i + 1]) - 1 for i in range(4)]
    out, lse = attend(cache, q[np_index(last)], scale, ints(rows), window, sink, layer=1)
    check(cache, q[np_index(last)], out, lse, scale, rows, window, sink, layer=1)
    for i in range(4):
        b = int(np.searchsorted(start, last[i], side="right")) - 1
        r = b * page + last[i] - int(start[b])
        tol = 2.0 ** -6 if dtype == "bf16" else 1e-4
        assert torch.allclose(ob[r].float(), out[i].float(), atol=tol, rtol=tol) and torch.allclose(lb[:, r], lse[:, i], atol=1e-3)
    # decoding; a place of the batch is padding
    kn, vn = (torch.empty((5, hkv, d), dtype=q.dtype, device="cuda") for _ in range(2))
    qn, on = torch.empty((5, hq, d), dtype=q.dtype, device="cuda"), torch.full((5, hq, d), NAN, dtype=q.dtype, device="cuda")
    ln = torch.full((hq, 5), NAN, dtype=torch.float32, device="cuda")
    ws = torch.empty(P.dcp_paged_attn_workspace_bytes(cache, 5, hq), dtype=torch.uint8, device="cuda").random_()

    def step():
        P.dcp_cache_reserve(cache, seqs, status)
        for layer in range(layers):
            P.dcp_cache_append(cache, kn, vn, seqs=seqs, status=status, layer=layer)
        P.dcp_paged_attn_fwd(cache, qn, on, ln, scale, ws, seqs=seqs, window=window, sink=sink, layer=1)

    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
    for t in range(steps):
        kn.copy_(K[1][0][T + 5 * t: T + 5 * t + 5])
        vn.copy_(K[1][1][T + 5 * t: T + 5 * t + 5])
        qn.copy_(randn((5, hq, d), dtype, 50 + t))
        if graph:
            g.replay()
        else:
            step()
        torch.cuda.synchronize()
        assert status.tolist() == [0] * 5
        assert cache.seq_len.cpu().numpy()[rows].tolist() == [n + t + 1 for n in prompts]
        check(cache, qn, on, ln, scale, rows + [-1], window, sink, layer=1)
    # the keys of the pages are those that went in
    for i, s in enumerate(rows):
        n = prompts[i] + steps
        at = cache.page_table[s, :-(-n // page)].long()
        want = torch.cat([K[1][0][int(cu[i]): int(cu[i + 1])], torch.stack([K[1][0][T + 5 * t + i] for t in range(steps)])])
        assert torch.equal(cache.k[1][at].flatten(0, 1)[:n], want)
    # a beam: two copies of a sequence go on from the same tokens, the others end
    st2 = ints([7, 7])
    P.dcp_cache_fork(cache, ints([4, 4]), ints([1, 3]), st2)
    P.dcp_cache_free(cache, ints([0, 5, 2]))
    counts, cws = ints([0, 0]), torch.empty(P.dcp_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    P.dcp_cache_compact(cache, counts, cws)
    assert st2.tolist() == [0, 0]
    tokens = prompts[0] + steps
    assert counts.tolist()[0] == tokens // page + 3 * (tokens % page != 0)
    P.dcp_cache_reserve(cache, ints([1, 3, 4]), ints([0, 0, 0]))
    P.dcp_cache_append(cache, kn[:3], vn[:3], seqs=ints([1, 3, 4]), layer=1)
    out, lse = attend(cache, qn[:3], scale, ints([1, 3, 4]), window, sink, layer=1)
    check(cache, qn[:3], out, lse, scale, [1, 3, 4], window, sink, layer=1)
    assert not torch.isnan(out).any()


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("dtype,d,window,sink", [("bf16", 128, 0, 0), ("bf16", 64, 40, 5), ("f32", 64, 0, 0)])
def test_prefill_decode_beam(dtype, d, window, sink, graph):
    _prefill_then_decode(dtype, d, graph, window, sink)


def test_on_a_stream_of_its_own_and_two_at_once():
    import torch
    cache, names = make_cache([500, 3000, 64], 16, 2, 128, seed=60)
    q = [randn((3, 8, 128), "bf16", 61 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.full_like(x, NAN) for x in q]
    lses = [torch.full((8, 3), NAN, dtype=torch.float32, device="cuda") for _ in q]
    spaces = [torch.empty(P.dcp_paged_attn_workspace_bytes(cache, 3, 8), dtype=torch.uint8, device="cuda") for _ in q]
    seqs = ints(names)
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                P.dcp_paged_attn_fwd(cache, q[i], outs[i], lses[i], 0.1, spaces[i], seqs=seqs)
    torch.cuda.synchronize()
    for i in range(2):
        check(cache, q[i], outs[i], lses[i], 0.1, [int(s) for s in names])


def test_two_graphs_share_a_workspace():
    """Calls of other sizes captured into two graphs over one workspace, replayed in turn with eager calls between them."""
    import torch
    cases = []
    ws = None
    for lens, hq in (([3000, 100, 17], 8), ([50, 700], 4)):
        cache, names = make_cache(lens, 16, 2, 64, seed=hq, width=300)
        q = randn((len(lens), hq, 64), "bf16", 71)
        out, lse = attend(cache, q, 0.1, ints(names))
        need = P.dcp_paged_attn_workspace_bytes(cache, len(lens), hq)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda").random_() if ws is None or ws.numel() < need else ws
        cases.append([cache, q, torch.full_like(out, NAN), torch.full_like(lse, NAN), ints(names), out, lse])
    graphs = []
    for cache, q, out, lse, seqs, _, _ in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            P.dcp_paged_attn_fwd(cache, q, out, lse, 0.1, ws, seqs=seqs)
        graphs.append(g)
    for _ in range(3):
        for g, (cache, q, out, lse, seqs, want, want_l) in zip(graphs, cases):
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(lse, want_l)
            out.fill_(NAN)
            lse.fill_(NAN)
            ws.random_()
            P.dcp_paged_attn_fwd(cache, q, out, lse, 0.1, ws, seqs=seqs)
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(lse, want_l)
            out.fill_(NAN)


def test_the_same_call_gives_the_same_bits():
    import torch
    cache, names = make_cache([5000, 300, 64, 9], 16, 2, 128, seed=62)
    q = randn((4, 8, 128), "bf16", 63)
    first = attend(cache, q, 0.1, ints(names))
    for _ in range(3):
        again = attend(cache, q, 0.1, ints(names))
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_binding_refuses():
    import torch
    cache, names = make_cache([30, 20], 8, 2, 64, seed=64)
    q, lse = randn((2, 4, 64), "bf16", 65), torch.empty((4, 2), dtype=torch.float32, device="cuda")
    ws = torch.empty(P.dcp_paged_attn_workspace_bytes(cache, 2, 4), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    ok = ints(names)
    for bad in (dict(seqs=ok.cpu()), dict(seqs=ok.long()), dict(seqs=ints([0])), dict(q=q.float()), dict(q=q.cpu()), dict(out=out[:1]), dict(lse=lse.t()),
                dict(lse=lse.double()), dict(ws=ws.cpu())):
        a = dict(q=q, out=out, lse=lse, ws=ws, seqs=ok)
        a.update(bad)
        with pytest.raises(ValueError):
            P.dcp_paged_attn_fwd(cache, a["q"], a["out"], a["lse"], 0.1, a["ws"], seqs=a["seqs"])
    with pytest.raises(P.DcpError) as ei:
        P.dcp_paged_attn_fwd(cache, q, q, lse, 0.1, ws, seqs=ok)
    assert ei.value.status == P.DCP_ERR_INVALID_ARG and "overlaps" in str(ei.value)
    for bad in (dict(k=cache.k[0]), dict(v=cache.v.float()), dict(page_ref=cache.page_ref[1:]), dict(seq_len=cache.seq_len.long()), dict(page_table=cache.page_table.t())):
        a = dict(k=cache.k, v=cache.v, page_ref=cache.page_ref, page_table=cache.page_table, seq_len=cache.seq_len)
        a.update(bad)
        with pytest.raises(ValueError):
            P.Cache(**a)
    with pytest.raises(ValueError):
        P.dcp_cache_append(cache, q[:, :2], q[:, :2], seqs=ints([0]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 32])
@pytest.mark.parametrize("hq,hkv", [(16, 1), (9, 3), (27, 3), (40, 1), (32, 8)])
@pytest.mark.parametrize("page", [20, 37, 64])
def test_wide_groups_in_any_pages(dtype, d, hq, hkv, page):
    cache, names = make_cache([1, 45, 700, 333], page, hkv, d, dtype, seed=hq + page)
    q = randn((4, hq, d), dtype, 75)
    out, lse = attend(cache, q, d ** -0.5, ints(names))
    check(cache, q, out, lse, d ** -0.5, [int(s) for s in names])
    out, lse = attend(cache, q, d ** -0.5, ints(names), 50, 10)
    check(cache, q, out, lse, d ** -0.5, [int(s) for s in names], 50, 10)


def test_places_without_seqs():
    """Reserve, append and attention where place i is sequence i."""
    import torch
    cache = P.Cache.empty(1, 20, 8, 2, 64, 5, 6, torch.bfloat16)
    cache.k.fill_(NAN)
    cache.v.fill_(NAN)
    m = mirror(cache)
    status = ints([7] * 4)
    new = [9, 0, 1, 30]
    P.dcp_cache_reserve(cache, None, status, n_new=ints(new))
    assert status.tolist() == m.reserve(range(4), new)
    k, v = randn((40, 2, 64), "bf16", 76), randn((40, 2, 64), "bf16", 77)
    P.dcp_cache_append(cache, k, v, cu_new=ints([0, 9, 9, 10, 40]))
    m.append(range(4), [0, 9, 9, 10, 40], words(k), words(v), [0] * 4)
    same_map(cache, m)
    P.dcp_cache_reserve(cache, None, status)
    assert status.tolist() == m.reserve(range(4), [1] * 4)
    P.dcp_cache_append(cache, k[:4], v[:4])
    m.append(range(4), [0, 1, 2, 3, 4], words(k), words(v), [0] * 4)
    same_map(cache, m)
    q = randn((5, 4, 64), "bf16", 78)
    out, lse = attend(cache, q, 0.125)
    check(cache, q, out, lse, 0.125, range(5))


def test_no_places_and_timing():
    """Calls without places do nothing; the calls are timed under ids of their own."""
    import torch
    cache, names = make_cache([30, 20], 8, 2, 64, seed=79)
    m = mirror(cache)
    none = ints([])
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    P.dcp_cache_reserve(cache, none, none)
    P.dcp_cache_append(cache, q[:, :2], q[:, :2], seqs=none)
    P.dcp_cache_fork(cache, none, none, none)
    P.dcp_cache_free(cache, none)
    P.dcp_paged_attn_fwd(cache, q, q.clone(), torch.empty((4, 0), device="cuda"), 0.1, torch.empty(0, dtype=torch.uint8, device="cuda"), seqs=none)
    same_map(cache, m)
    P.dcp_profile_enable(True)
    attend(cache, randn((2, 4, 64), "bf16", 80), 0.1, ints(names))
    P.dcp_cache_free(cache, ints(names))
    (ms, n), (ms_c, n_c) = P.dcp_profile_read("paged_attn"), P.dcp_profile_read("cache")
    P.dcp_profile_enable(False)
    assert n == n_c == 1 and 0 < ms < 100 and 0 < ms_c < 100


def test_a_captured_life_of_a_cache():
    """Fork, free and compaction recorded once and replayed on the map as it is each time, with eager calls between, against the oracle."""
    import torch
    cache, names = make_cache([20, 33, 7], 8, 2, 32, layers=2, spare=20, extra_seqs=5, width=12, seed=81)
    m = mirror(cache)
    a, b, c = (int(s) for s in names)
    empty = [s for s in range(8) if s not in (a, b, c)]
    src, dst, gone = [a, b, -1], [empty[0], empty[1], empty[2]], [a, 99]
    args = ints(src), ints(dst), ints([7] * 3), ints(gone), ints([0, 0])
    ws = torch.empty(P.dcp_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda").random_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.dcp_cache_fork(cache, args[0], args[1], args[2])
        P.dcp_cache_free(cache, args[3])
        P.dcp_cache_compact(cache, args[4], ws)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        want = m.fork(src, dst)
        m.free(gone)
        assert args[4].tolist() == m.compact() and args[2].tolist() == want
        same_map(cache, m)
        ws.random_()
        # another life between: the copies end, the source fills again
        P.dcp_cache_free(cache, ints(dst[:2]))
        m.free(dst[:2])
        status = reserve(cache, m, [a], [13])
        append(cache, m, [a], [13], status, 1, 82)
        same_map(cache, m)
