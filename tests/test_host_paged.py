"""Refusals of the calls on a paged cache: every one is the host's, before any launch, so that they run without a GPU
(the addresses are never followed)."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2510_10620_amd as P
from paper_2510_10620_amd import _lib

A = 0x10000   # a 256-byte aligned address


def _cache(**kw):
    c = _lib.Cache()
    c.n_layers, c.n_pages, c.page_size, c.hkv, c.d, c.dtype, c.n_seqs, c.max_pages = 2, 10, 16, 2, 64, P.DCP_BF16, 5, 4
    for n in "kv":
        setattr(c, n, A)
        for letter, x in zip("lpth", (10 * 16 * 128, 16 * 128, 128, 64)):
            setattr(c, f"{n}_stride_{letter}", x)
    c.page_ref = c.page_table = c.seq_len = A
    for name, x in kw.items():
        setattr(c, name, x)
    return c


def _attn(**kw):
    a = _lib.PagedAttn()
    a.n, a.hq, a.layer, a.softmax_scale = 3, 4, 0, 0.5
    a.seqs, a.q, a.out, a.lse = A, A, A << 4, A
    a.q_stride_t, a.q_stride_h, a.o_stride_t, a.o_stride_h = 256, 64, 256, 64
    for name, x in kw.items():
        setattr(a, name, x)
    return a


def _ref(c):
    return ctypes.byref(c)


BAD_CACHES = [(dict(n_layers=0), -1), (dict(n_pages=0), -1), (dict(page_size=-1), -1), (dict(hkv=0), -1), (dict(n_seqs=0), -1), (dict(max_pages=0), -1),
              (dict(dtype=2), -4), (dict(d=96), -4), (dict(n_seqs=16385), -4), (dict(n_pages=(1 << 30) + 1), -4),
              (dict(max_pages=1 << 16, page_size=1 << 15), -4), (dict(k=0), -1), (dict(v=A + 8), -1), (dict(k_stride_t=56), -1),
              (dict(v_stride_p=0), -1), (dict(k_stride_l=4), -1), (dict(v_stride_h=68), -1), (dict(page_ref=0), -1), (dict(page_table=A + 2), -1),
              (dict(seq_len=0), -1), (dict(page_size=1 << 24, max_pages=1), -4)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(kw, status):
    lib, c = _lib.load(), _cache(**kw)
    assert lib.dcp_cache_reserve(_ref(c), A, None, 3, A, None) == status
    assert lib.dcp_cache_append(_ref(c), 0, A, None, 3, None, A, 128, 64, A, 128, 64, 3, None) == status
    assert lib.dcp_cache_fork(_ref(c), A, A, 3, A, None) == status
    assert lib.dcp_cache_free(_ref(c), A, 3, None) == status
    assert lib.dcp_cache_compact(_ref(c), A, A, 1 << 40, None) == status
    assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn()), A, 1 << 40, None) == status
    assert P.dcp_last_error()


def test_reserve_fork_free_compact_refuse():
    lib, c = _lib.load(), _cache()
    for n, seqs, status, want in ((-1, A, A, -1), (16385, A, A, -4), (6, None, A, -1), (3, A, None, -1), (3, A, A + 1, -1), (3, A + 2, A, -1)):
        assert lib.dcp_cache_reserve(_ref(c), seqs, None, n, status, None) == want
    assert lib.dcp_cache_reserve(_ref(c), A, A + 1, 3, A, None) == -1
    assert lib.dcp_cache_fork(_ref(c), None, A, 3, A, None) == -1
    assert lib.dcp_cache_fork(_ref(c), A, None, 3, A, None) == -1
    assert lib.dcp_cache_fork(_ref(c), A, A, 3, None, None) == -1
    assert lib.dcp_cache_fork(_ref(c), A, A, 16385, A, None) == -4
    assert lib.dcp_cache_free(_ref(c), None, 6, None) == -1
    assert lib.dcp_cache_free(_ref(c), A, -2, None) == -1
    need = lib.dcp_cache_workspace_bytes(_ref(c))
    assert need > 0 and lib.dcp_cache_workspace_bytes(None) == 0
    assert lib.dcp_cache_compact(_ref(c), None, A, need, None) == -1
    assert lib.dcp_cache_compact(_ref(c), A, None, need, None) == -5
    assert lib.dcp_cache_compact(_ref(c), A, A, need - 1, None) == -5
    assert lib.dcp_cache_compact(_ref(c), A, A + 16, need, None) == -5
    # nothing to do is legal
    assert lib.dcp_cache_reserve(_ref(c), None, None, 0, None, None) == 0
    assert lib.dcp_cache_fork(_ref(c), None, None, 0, None, None) == 0
    assert lib.dcp_cache_free(_ref(c), None, 0, None) == 0
    assert lib.dcp_cache_append(_ref(c), 0, None, None, 0, None, None, 0, 0, None, 0, 0, 0, None) == 0
    assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn(n=0)), None, 0, None) == 0


def test_append_refuses():
    lib, c = _lib.load(), _cache()
    good = dict(layer=0, seqs=A, cu=None, n=3, status=None, k=A, kt=128, kh=64, v=A, vt=128, vh=64, n_tokens=3)
    for kw, want in ((dict(layer=2), -1), (dict(layer=-1), -1), (dict(n=-1), -1), (dict(k=None), -1), (dict(v=A + 8), -1), (dict(kt=63), -1),
                     (dict(vh=68), -1), (dict(n_tokens=-1), -1), (dict(n_tokens=(1 << 26) + 1), -4), (dict(cu=A + 1), -1), (dict(status=A + 2), -1)):
        x = dict(good, **kw)
        assert lib.dcp_cache_append(_ref(c), x["layer"], x["seqs"], x["cu"], x["n"], x["status"], x["k"], x["kt"], x["kh"], x["v"], x["vt"], x["vh"],
                                    x["n_tokens"], None) == want, kw


def test_append_refuses_more_tokens_than_a_grid_has_threads_for():
    lib, c = _lib.load(), _cache()
    for n_tokens in ((1 << 25) + 1, (1 << 26) - 3, 1 << 26):
        assert lib.dcp_cache_append(_ref(c), 0, A, A, 3, None, A, 128, 64, A, 128, 64, n_tokens, None) == -4 and "2^25" in P.dcp_last_error()


def test_attention_refuses():
    lib, c = _lib.load(), _cache()
    need = lib.dcp_paged_attn_workspace_bytes(_ref(c), 3, 4)
    assert need > 0 and lib.dcp_paged_attn_workspace_bytes(None, 3, 4) == 0
    nan = float("nan")
    for kw, want in ((dict(n=-1), -1), (dict(n=16385), -4), (dict(seqs=0, n=6), -1), (dict(hq=0), -1), (dict(hq=3), -4), (dict(layer=2), -1),
                     (dict(softmax_scale=0.0), -1), (dict(softmax_scale=nan), -1), (dict(softmax_scale=float("inf")), -1), (dict(window=-1), -1),
                     (dict(sink=-1), -1), (dict(q=0), -1), (dict(q=A + 4), -1), (dict(out=0), -1), (dict(lse=0), -1), (dict(lse=A + 2), -1),
                     (dict(q_stride_t=63), -1), (dict(o_stride_h=60), -1), (dict(out=A + 64), -1)):
        assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn(**kw)), A, max(need, 1 << 30), None) == want, kw
    full = _cache(max_pages=1 << 26)   # 2^30 tokens a row: 16 384 places of 2^25 tiles
    assert lib.dcp_paged_attn_fwd(_ref(full), ctypes.byref(_attn(n=16384, out=A << 20)), A, 1 << 30, None) == -4 and "2^31" in P.dcp_last_error()
    assert lib.dcp_paged_attn_fwd(_ref(c), None, A, need, None) == -1
    assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn()), None, need, None) == -5
    assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn()), A, need - 1, None) == -5
    assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn()), A + 128, need, None) == -5


@pytest.mark.parametrize("hkv,hq", [(1, 2 ** 31 - 1), (1, 2 ** 31 - 15), (2, 2 ** 31 - 2), (2, 2 ** 17 + 2)])
def test_attention_refuses_more_heads_than_it_can_count(hkv, hq):
    """Sets of heads whose sums would leave 32 bits, and whose products with places and tiles 64."""
    lib = _lib.load()
    for c, n in ((_cache(hkv=hkv), 3), (_cache(hkv=hkv, max_pages=1 << 26), 16384)):
        assert lib.dcp_paged_attn_workspace_bytes(_ref(c), n, hq) > 0
        assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn(hq=hq, n=n, out=1 << 62, o_stride_t=64)), A, 1 << 40, None) == -4
        assert "4 096" in P.dcp_last_error()


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_index_arithmetic_of_the_kernels(tmp_path):
    """csrc/paged.h on the CPU, under the undefined-behaviour sanitizer: tests/host_paged/driver.cpp."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "host_paged")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-I" + os.path.join(root, "include"),
                        "-I" + os.path.join(root, "paper_2510_10620_amd", "csrc"), os.path.join(root, "tests", "host_paged", "driver.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "host-paged ok" in r.stdout, r.stdout[-2000:] + r.stderr[-3000:]
