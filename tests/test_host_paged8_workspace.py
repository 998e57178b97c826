"""The workspace of dcp_paged_attn_chunk_fwd: one that was taken for the largest batch does for every smaller one.  No GPU."""
import ctypes
import itertools

import pytest

import paper_2510_10620_amd as P
from paper_2510_10620_amd import _lib
from tests.test_host_paged import A, _attn, _ref
from tests.test_host_paged8 import _cache8

PLACES, TOKENS = [1, 2, 3, 16, 48, 64, 128, 200, 1000, 16384], [1, 2, 5, 31, 32, 33, 63, 320, 512, 513, 1024, 5000, 70000, 1 << 25]


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (4, 2, 64), (1, 1, 32), (64, 2, 64), (16, 1, 128), (24, 24, 32), (4000, 1, 64)])
def test_workspace_grows_with_places_and_tokens(hq, hkv, d):
    lib, c = _lib.load(), _cache8(hkv=hkv, d=d, k_stride_h=d, v_stride_h=d, k_stride_t=hkv * d, v_stride_t=hkv * d)
    size = {(n, t): lib.dcp_paged_attn_chunk_workspace_bytes(_ref(c), n, t, hq) for n in PLACES for t in TOKENS}
    for (n, t), bytes_ in size.items():
        assert bytes_ > 0
        assert all(size[m, u] <= bytes_ for m, u in itertools.product(PLACES, TOKENS) if m <= n and u <= t), (n, t)


@pytest.mark.parametrize("n,tokens", [(64, 320), (128, 512), (1, 512), (5, 32), (1, 1)])
def test_a_workspace_of_the_largest_batch_does_for_smaller_ones(n, tokens):
    """Up to the check of the address, which comes behind that of the size."""
    lib, c = _lib.load(), _cache8(hkv=8, d=128, k_stride_t=1024, v_stride_t=1024, k_stride_h=128, v_stride_h=128)
    most = lib.dcp_paged_attn_chunk_workspace_bytes(_ref(c), n, tokens, 32)
    for m, u in itertools.product(sorted({1, 2, n // 2 or 1, n}), sorted({1, 8, 33, 100, tokens // 2 or 1, tokens})):
        if m > n or u > tokens:
            continue
        args = ctypes.byref(_attn(n=m, hq=32, q_stride_t=4096, q_stride_h=128, o_stride_t=4096, o_stride_h=128, out=1 << 40))
        assert lib.dcp_paged_attn_chunk_fwd(_ref(c), args, A, u, A + 128, most, None) == -5
        assert "aligned" in P.dcp_last_error(), (m, u, P.dcp_last_error())
