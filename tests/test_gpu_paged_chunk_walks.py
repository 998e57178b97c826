"""Attention of the last tokens of every place in both of its walks, with the keys in registers and in LDS, beside the attention of one token: what has to
come out alike whichever walk the rest of the batch leads to."""
import numpy as np
import pytest

import paper_2510_10620_amd as P
from tests.paged8 import NAN, Held, f64, infinite_at, ints, make_cache, randn
from tests.test_gpu_paged_chunk import BOTH, chunk

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
