"""Arithmetic of the calls on a paged cache at the limits that the host accepts, on the CPU under the undefined-behaviour sanitizer."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2510_10620_amd as P
from paper_2510_10620_amd import _lib
from tests.test_host_paged import A, _attn, _cache, _ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(tmp_path, name):
    """tests/host_paged/<name>.cpp, which says "host-paged <name> ok"."""
    exe = str(tmp_path / name)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-I" + os.path.join(ROOT, "include"),
                        "-I" + os.path.join(ROOT, "paper_2510_10620_amd", "csrc"), os.path.join(ROOT, "tests", "host_paged", name + ".cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and f"host-paged {name} ok" in r.stdout, r.stdout[-2000:] + r.stderr[-3000:]


gxx = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@gxx
def test_sums_of_needs_up_to_the_most_pages(tmp_path):
    _run(tmp_path, "sums")


@gxx
def test_queries_and_outputs_that_share_bytes(tmp_path):
    _run(tmp_path, "overlap")


def test_attention_refuses_a_misaligned_status():
    assert _lib.load().dcp_paged_attn_fwd(_ref(_cache()), ctypes.byref(_attn(status=A + 2)), A, 1 << 30, None) == P.DCP_ERR_INVALID_ARG
    assert "status" in P.dcp_last_error()


FAR = (1 << 58) + 8


@pytest.mark.parametrize("kw", [dict(n_layers=65537), dict(n_layers=2 ** 31 - 1), dict(k_stride_l=FAR), dict(v_stride_p=FAR), dict(k_stride_t=2 ** 63 - 8), dict(v_stride_h=FAR)])
def test_every_call_refuses_what_64_bits_cannot_count(kw):
    """Layers times pages times pieces of a page; strides in bytes."""
    lib, c = _lib.load(), _cache(**kw)
    for got in (lib.dcp_cache_reserve(_ref(c), A, None, 3, A, None), lib.dcp_cache_append(_ref(c), 0, A, None, 3, None, A, 128, 64, A, 128, 64, 3, None),
                lib.dcp_cache_fork(_ref(c), A, A, 3, A, None), lib.dcp_cache_free(_ref(c), A, 3, None), lib.dcp_cache_compact(_ref(c), A, A, 1 << 40, None),
                lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn()), A, 1 << 30, None)):
        assert got == P.DCP_ERR_UNSUPPORTED and ("65 536" in P.dcp_last_error() or "2^58" in P.dcp_last_error())


def test_rows_beside_the_cache_refuse_strides_that_64_bits_cannot_count():
    lib, c = _lib.load(), _cache()
    for st, sh in ((FAR, 64), (128, FAR)):
        assert lib.dcp_cache_append(_ref(c), 0, A, None, 3, None, A, st, sh, A, 128, 64, 3, None) == P.DCP_ERR_UNSUPPORTED
        assert lib.dcp_cache_append(_ref(c), 0, A, None, 3, None, A, 128, 64, A, st, sh, 3, None) == P.DCP_ERR_UNSUPPORTED
        assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn(q_stride_t=st, q_stride_h=sh)), A, 1 << 30, None) == P.DCP_ERR_UNSUPPORTED
        assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn(o_stride_t=st, o_stride_h=sh)), A, 1 << 30, None) == P.DCP_ERR_UNSUPPORTED
