"""Places that dcp_cache_reserve refused, in the calls that follow: append leaves them out, and so does attention."""
import numpy as np
import pytest

import paper_2510_10620_amd as P
from oracle import paged as OP
from tests.test_gpu_paged import NAN, attend, check, ints, make_cache, mirror, randn, same_map, words

pytestmark = pytest.mark.gpu


def _attend(cache, q, out, lse, scale, ws, seqs, status, **kw):
    P.dcp_paged_attn_fwd(cache, q, out, lse, scale, ws, seqs=seqs, status=status, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,width", [(1, None), (5, None), (40, 300), (300, 300), (600, 300)])
def test_places_that_are_not_ok_are_padding(dtype, n, width):
    """Items taken whole, cut with an entry of the joins an item, cut with one a worker; several places a thread.  What is left is as if
    the others were not there, to the last bit."""
    import torch
    rng = np.random.default_rng(n)
    cache, names = make_cache([int(x) for x in rng.integers(1, 200, n)], 16, 2, 64, dtype, seed=n, width=width)
    codes = [int(x) for x in rng.integers(0, 3, n)]
    codes[0] = OP.FULL
    q = randn((n, 8, 64), dtype, 1)
    ws = torch.empty(P.dcp_paged_attn_workspace_bytes(cache, n, 8), dtype=torch.uint8, device="cuda").random_()
    left = [int(s) if code == OP.OK else -1 for s, code in zip(names, codes)]
    for window, sink in ((0, 0), (20, 3)):
        want, want_l = attend(cache, q, 0.125, ints(left), window, sink)
        out, lse = torch.full_like(q, NAN), torch.full((8, n), NAN, dtype=torch.float32, device="cuda")
        _attend(cache, q, out, lse, 0.125, ws, ints(names), ints(codes), window=window, sink=sink)
        torch.cuda.synchronize()
        check(cache, q, out, lse, 0.125, left, window, sink)
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want)) and torch.equal(torch.nan_to_num(lse), torch.nan_to_num(want_l))


def test_place_i_is_sequence_i_where_it_is_ok():
    import torch
    cache, _ = make_cache([70, 1, 333, 50], 32, 1, 128, extra_seqs=0, seed=8)
    q, ws = randn((4, 4, 128), "bf16", 6), torch.empty(P.dcp_paged_attn_workspace_bytes(cache, 4, 4), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, NAN), torch.full((4, 4), NAN, dtype=torch.float32, device="cuda")
    _attend(cache, q, out, lse, 0.1, ws, None, ints([0, 1, 2, 0]))
    torch.cuda.synchronize()
    check(cache, q, out, lse, 0.1, [0, -1, -1, 3])


@pytest.mark.parametrize("graph", [False, True])
def test_steps_in_which_pages_run_out(graph):
    """A decoding step, captured or not, while pages run out, a sequence is named twice and a row of the table is full: places without room write
    nothing, the others go on; when pages are given back all do."""
    import torch
    cache, names = make_cache([15, 16, 7, 31, 47], 8, 2, 64, layers=2, spare=2, extra_seqs=0, width=6, seed=3)
    m = mirror(cache)
    rows = [int(s) for s in names]
    places = rows + [rows[2], -1, 99]
    n = len(places)
    seqs, status = ints(places), ints([7] * n)
    kn, vn = (torch.empty((n, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out, lse = torch.empty((n, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((n, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((4, n), device="cuda")
    ws = torch.empty(P.dcp_paged_attn_workspace_bytes(cache, n, 4), dtype=torch.uint8, device="cuda").random_()

    def step():
        P.dcp_cache_reserve(cache, seqs, status)
        for layer in range(2):
            P.dcp_cache_append(cache, kn, vn, seqs=seqs, status=status, layer=layer)
        _attend(cache, q, out, lse, 0.125, ws, seqs, status, layer=1)

    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
    seen = set()
    for t in range(10):
        if t == 7:
            P.dcp_cache_free(cache, ints([rows[4]]))
            m.free([rows[4]])
        for i, x in enumerate((kn, vn, q)):
            x.copy_(randn(x.shape, "bf16", 10 * t + i))
        out.fill_(NAN)
        lse.fill_(NAN)
        g.replay() if graph else step()
        torch.cuda.synchronize()
        want = m.reserve(places, [1] * n)
        for layer in range(2):
            m.append(places, list(range(n + 1)), words(kn), words(vn), want, layer)
        assert status.tolist() == want
        same_map(cache, m)
        check(cache, q, out, lse, 0.125, [s if code == OP.OK else -1 for s, code in zip(places, want)], layer=1)
        seen.update(want)
    assert seen == {OP.OK, OP.FULL, OP.BAD} and want[:4].count(OP.OK) == 4


def test_status_of_another_size_or_place_is_refused():
    import torch
    cache, names = make_cache([30, 20], 8, 2, 64, seed=64)
    q, lse = randn((2, 4, 64), "bf16", 65), torch.empty((4, 2), dtype=torch.float32, device="cuda")
    ws = torch.empty(P.dcp_paged_attn_workspace_bytes(cache, 2, 4), dtype=torch.uint8, device="cuda")
    for status in (ints([0]), ints([0, 0]).cpu(), ints([0, 0]).long()):
        with pytest.raises(ValueError):
            _attend(cache, q, torch.empty_like(q), lse, 0.1, ws, ints(names), status)
