"""Attention of the last tokens of every place in both of its walks, with the keys in registers and in LDS, beside the attention of one token: what has to
come out alike whichever walk the rest of the batch leads to."""
import numpy as np
import pytest

import paper_2510_10620_amd as P
from tests.paged8 import NAN, Held, check_rows, f64, infinite_at, ints, make_cache, randn
from tests.test_gpu_paged_chunk import BOTH, WEIGHTS, chunk, rows_of

pytestmark = pytest.mark.gpu


def attend(cache, q, scale, seqs):
    import torch
    out, lse = torch.full_like(q, NAN), torch.full((q.shape[1], q.shape[0]), NAN, dtype=torch.float32, device="cuda")
    ws = torch.empty(P.dcp_paged_attn_workspace_bytes(cache, q.shape[0], q.shape[1]), dtype=torch.uint8, device="cuda")
    P.dcp_paged_attn_fwd(cache, q, out, lse, scale, ws, seqs=seqs)
    return out, lse


@pytest.mark.parametrize("io,d", [("bf16", 128), ("bf16", 32), ("f32", 64)])
@pytest.mark.parametrize("page,block,pos", [(16, 16, 85), (20, 10, 110), (8, 8, 81), (48, 16, 250)])
@pytest.mark.parametrize("n", [300, 5000])
@BOTH
def test_nan_and_infinity_beside_a_page_that_does_not_exist(io, d, page, block, pos, n, in_lds):
    """All rows see the key at `pos`; the page before its own, which shares a tile of 32 keys with it, is missing."""
    import torch
    cache, names = make_cache([n, n], page, block, 1, d, io)
    a, b = (int(s) for s in names)
    assert pos // 32 == pos // page * page // 32 and pos // page * page % 32
    cache.page_table[a, pos // page - 1], cache.page_table[b, pos // page - 1] = -1, 10 ** 6
    v = cache.v.view(torch.uint8)
    p, slot = infinite_at(cache, b, pos)
    cache.k.view(torch.uint8)[0, p, slot] = 0
    at = (0, int(cache.page_table[a, pos // page]), pos % page, 0)
    places, cu = ints([a, b]), [0, 8, 16]
    q = randn((16, 4, d), io, 1)
    last = torch.stack([q[7], q[15]])
    got = []
    for nan, inf in ((0x7f, 0x7e), (0, 0)):
        v[(*at, 7)], v[0, p, slot, 0, 3], v[0, p, slot, 0, 4] = nan, inf, inf | 0x80
        out, lse = chunk(cache, q, d ** -0.5, cu, places, in_lds=in_lds)
        o1, l1 = attend(cache, last, d ** -0.5, places)
        got.append([f64(x) for x in (out, lse, o1, l1)])
    (out, lse, o1, l1), clean = got
    assert np.isfinite(lse).all() and np.array_equal(lse, clean[1]) and np.array_equal(l1, clean[3])
    for o, c, rows in ((out, clean[0], 8), (o1, clean[2], 1)):
        assert np.isfinite(c).all()
        assert np.isnan(o[:rows, :, 7]).all() and (o[rows:, :, 3] == np.inf).all() and (o[rows:, :, 4] == -np.inf).all()
        assert np.array_equal(np.delete(o[:rows], 7, 2), np.delete(c[:rows], 7, 2)) and np.array_equal(np.delete(o[rows:], [3, 4], 2), np.delete(c[rows:], [3, 4], 2))


@pytest.mark.parametrize("io,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("n", [100, 3000])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("scale", [0.088, 0.0613, 0.3])
@BOTH
def test_scores_of_2_to_the_31_and_more(io, d, n, sign, scale, in_lds):
    """All keys are alike, so that all weights are, whatever a score of this size is rounded to: O is the mean of the values, to the bits of the weights (rounded
    to 2^-8 at most), of their sums and of the output; the LSE is the score, after a rounding of each of scale, log2 e, their product, the score's and the way back."""
    import torch
    cache, names = make_cache([n], 16, 16, 1, d, io)
    cache.k.view(torch.uint8)[0, cache.page_table[int(names[0])].long()] = 0x3b   # 1.375
    cache.k_scale[:] = 127 + 15
    q = randn((8, 2, d), io, 1).fill_(sign * 2.0 ** 15 * 1.171875)
    v = Held(cache).values(int(names[0]), np.arange(n))[2][:, 0]
    score = sign * d * 2.0 ** 30 * 1.375 * 1.171875 * float(np.float32(scale))
    out, lse = chunk(cache, q, scale, [0, 8], ints(names), in_lds=in_lds)
    o1, l1 = attend(cache, q[7:], scale, ints(names))
    for o, l, keys in [(f64(out)[i], f64(lse)[:, i], n - 7 + i) for i in range(8)] + [(f64(o1)[0], f64(l1)[:, 0], n)]:
        ref, mean = v[:keys].mean(0), np.abs(v[:keys]).mean(0)
        assert (np.abs(o - ref) <= (2.0 ** -8 if io == "bf16" else 2.0 ** -24) * np.abs(ref) + 1.01 * (2.0 ** -8 * (io == "bf16") + 2 * keys * 2.0 ** -24) * mean).all()
        assert (np.abs(l - score) <= 8 * 2.0 ** -24 * abs(score)).all()


# Walks, by the new tokens of the places and places that are padding: keys in LDS; in registers, with the items listed by the walk; by the launch before it, more than 256
WALKS = pytest.mark.parametrize("new,pad", [([60, 80, 50, 5, 90], 0), ([5, 4, 3, 2, 6], 0), ([5, 4, 3, 2, 6], 300)], ids=["lds", "registers", "listed_before"])


@pytest.mark.parametrize("io,d", [("bf16", 128), ("bf16", 32), ("f32", 64)])
@pytest.mark.parametrize("page,block", [(16, 16), (20, 10)])
@WALKS
def test_status_pages_and_rows_that_do_not_exist_in_every_walk(io, d, page, block, new, pad):
    lens = [200, 200, 200, 64, 180]
    cache, names = make_cache(lens, page, block, 2, d, io)
    a, b, c, _, _ = (int(s) for s in names)
    cache.page_table[a, 1], cache.page_table[a, 7], cache.page_table[b, :] = -1, 10 ** 6, -5
    places = [int(s) for s in names] + [1000] + [-1] * pad
    cu = (4 + np.concatenate([[0], np.cumsum(new + [3] + [0] * pad)])).tolist()
    q = randn((cu[5] - 2, 8, d), io, 7)                     # the last rows of the fifth place, and the sixth's, are not there
    out, lse = chunk(cache, q, 0.1, cu, ints(places), status=ints([0, 0, 1, 0, 0, 0] + [0] * pad))
    rows = rows_of([int(x) if s != c else 0 for s, x in enumerate(cache.seq_len.tolist())], places, cu, q.shape[0])
    assert [r for r in rows if r[1] == b]                   # of which no key exists
    check_rows(cache, q, out, lse, 0.1, rows, weights=WEIGHTS)


@WALKS
def test_graphs_and_streams_in_every_walk(new, pad):
    """Two caches' calls on two streams, then recorded into graphs that share a workspace and replayed in any order with other work between: the eager call's bits."""
    import torch
    lens = [500, 70, 1300, 8, 2000]
    made = [make_cache(lens, 32, 16, 2, 64, seed=s) for s in (1, 2)]
    cu = np.concatenate([[0], np.cumsum(new + [0] * pad)]).tolist()
    places = [[int(s) for s in names] + [-1] * pad for _, names in made]
    q = [randn((cu[-1], 8, 64), "bf16", s) for s in (3, 4)]
    want = [chunk(c, x, 0.125, cu, ints(p)) for (c, _), x, p in zip(made, q, places)]
    for (c, _), x, p, (o, l) in zip(made, q, places, want):
        check_rows(c, x, o, l, 0.125, rows_of(c.seq_len.tolist(), p, cu, cu[-1]), weights=WEIGHTS)
    size = P.dcp_paged_attn_chunk_workspace_bytes(made[0][0], len(cu) - 1, cu[-1], 8)
    got, args = [tuple(torch.full_like(x, NAN) for x in w) for w in want], [(ints(cu), ints(p)) for p in places]
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def call(i, space):
        P.dcp_paged_attn_chunk_fwd(made[i][0], q[i], *got[i], 0.125, space, args[i][0], seqs=args[i][1])

    def bits(x):                      # rows of positions below 0 hold NaN
        return x.view(torch.int16 if x.element_size() == 2 else torch.int32)

    def same():
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(bits(g[0]), bits(w[0])) and torch.equal(bits(g[1]), bits(w[1]))
            g[0].fill_(NAN)
            g[1].fill_(NAN)
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                call(i, spaces[i])
    same()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            call(i, spaces[0])
    for order in ((0, 1), (1, 0, 1), (0, 0, 1), (1, 0)):
        for i in order:
            graphs[i].replay()
        same()
        assert float(torch.ones(1 << 20, device="cuda").sum()) == 1 << 20
        call(0, spaces[0])
        torch.cuda.synchronize()
        assert torch.equal(bits(got[0][0]), bits(want[0][0]))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 32])
@pytest.mark.parametrize("page,block", [(16, 16), (20, 10), (64, 4)])
def test_weights_of_few_tokens_are_held_as_those_of_one(io, d, page, block):
    """In registers a weight in bf16 is held to 2^-15 of itself: the bound of one token."""
    lens, new = [1, 2, 31, 33, 64, 100, 300, 1000, 5000], [1, 2, 5, 4, 8, 3, 6, 3, 2]
    cache, names = make_cache(lens, page, block, 2, d, io, seed=page)
    places, cu = [int(s) for s in names], np.concatenate([[0], np.cumsum(new)]).tolist()
    q = randn((cu[-1], 8, d), io, 1)
    out, lse = chunk(cache, q, d ** -0.5, cu, ints(places))
    check_rows(cache, q, out, lse, d ** -0.5, rows_of(cache.seq_len.tolist(), places, cu, cu[-1]))
