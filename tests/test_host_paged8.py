"""Refusals of the calls on a paged cache in 8 bits, of dcp_cache_read and of dcp_paged_attn_chunk_fwd (the host's, before any launch: no address is followed),
and the host's code and the index arithmetic under sanitizers.  No GPU."""
import ctypes
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

import paper_2510_10620_amd as P
from paper_2510_10620_amd import _lib
from tests.test_host_asan import CSRC, FLAGS, HERE
from tests.test_host_paged import A, BAD_CACHES, _attn, _cache, _ref


def _cache8(**kw):
    x = dict(dtype=P.DCP_E4M3, io_dtype=P.DCP_BF16, scale_block=8, k_scale=A, v_scale=A)
    x.update(kw)
    return _cache(**x)


BAD_8 = [(dict(io_dtype=3), -4), (dict(io_dtype=2), -4), (dict(io_dtype=-1), -4), (dict(scale_block=0), -1), (dict(scale_block=-8), -1), (dict(scale_block=3), -1),
         (dict(scale_block=32), -1), (dict(k_scale=0), -1), (dict(v_scale=0), -1), (dict(k_stride_t=136), -1), (dict(v_stride_h=72), -1)]


@pytest.mark.parametrize("kw,status", BAD_8 + [x for x in BAD_CACHES if "dtype" not in x[0] and "page_size" not in x[0]])
def test_every_call_refuses_a_bad_cache(kw, status):
    lib, c = _lib.load(), _cache8(**kw)
    assert lib.dcp_cache_reserve(_ref(c), A, None, 3, A, None) == status
    assert lib.dcp_cache_append(_ref(c), 0, A, None, 3, None, A, 128, 64, A, 128, 64, 3, None) == status
    assert lib.dcp_cache_read(_ref(c), 0, A, None, 3, None, A, 128, 64, A << 4, 128, 64, 3, None) == status
    assert lib.dcp_cache_fork(_ref(c), A, A, 3, A, None) == status
    assert lib.dcp_cache_free(_ref(c), A, 3, None) == status
    assert lib.dcp_cache_compact(_ref(c), A, A, 1 << 40, None) == status
    assert lib.dcp_paged_attn_fwd(_ref(c), ctypes.byref(_attn()), A, 1 << 40, None) == status
    assert lib.dcp_paged_attn_chunk_fwd(_ref(c), ctypes.byref(_attn()), A, 6, A, 1 << 40, None) == status
    assert P.dcp_last_error()


def test_the_other_calls_take_no_numbers_in_8_bits():
    lib, t = _lib.load(), _lib.Tensors()
    t.hq, t.hkv, t.d, t.dtype, t.softmax_scale = 4, 2, 64, P.DCP_E4M3, 0.5
    assert lib.dcp_bwd_delta(ctypes.byref(t), 16, A, None) == -4
    parts = (ctypes.c_void_p * 1)(A)
    assert lib.dcp_sum_partials(parts, 1, P.DCP_E4M3, A, P.DCP_F32, 16, None) == -4


@pytest.mark.parametrize("cache", [_cache, _cache8])
def test_read_refuses(cache):
    lib, c = _lib.load(), cache()
    good = dict(layer=0, seqs=A, cu=None, n=3, status=None, k=A, kt=128, kh=64, v=A << 4, vt=128, vh=64, n_tokens=3)
    for kw, want in ((dict(layer=2), -1), (dict(layer=-1), -1), (dict(n=-1), -1), (dict(n=16385), -4), (dict(seqs=None, n=6), -1), (dict(seqs=A + 2), -1),
                     (dict(k=None), -1), (dict(v=A + 8), -1), (dict(kt=63), -1), (dict(vh=68), -1), (dict(kt=1 << 59), -4), (dict(n_tokens=-1), -1),
                     (dict(n_tokens=(1 << 25) + 1), -4), (dict(cu=A + 1), -1), (dict(status=A + 2), -1), (dict(v=A), -1), (dict(v=A + 256), -1)):
        x = dict(good, **kw)
        assert lib.dcp_cache_read(_ref(c), x["layer"], x["seqs"], x["cu"], x["n"], x["status"], x["k"], x["kt"], x["kh"], x["v"], x["vt"], x["vh"],
                                  x["n_tokens"], None) == want, kw
    assert lib.dcp_cache_read(_ref(c), 0, None, None, 0, None, None, 0, 0, None, 0, 0, 0, None) == 0
    assert lib.dcp_cache_read(_ref(c), 0, A, A, 3, None, None, 0, 0, None, 0, 0, 0, None) == 0


def test_chunk_refuses():
    lib, c = _lib.load(), _cache8()
    size = lib.dcp_paged_attn_chunk_workspace_bytes
    need = size(_ref(c), 3, 6, 4)
    assert need > 0 and size(None, 3, 6, 4) == 0 and size(_ref(c), 0, 6, 4) == 0 and size(_ref(c), 3, 0, 4) == 0 and size(_ref(c), 3, 6, 3) == 0
    nan, go = float("nan"), lib.dcp_paged_attn_chunk_fwd
    for kw, want in ((dict(n=-1), -1), (dict(n=16385), -4), (dict(seqs=0, n=6), -1), (dict(hq=0), -1), (dict(hq=3), -4), (dict(layer=2), -1),
                     (dict(softmax_scale=0.0), -1), (dict(softmax_scale=nan), -1), (dict(softmax_scale=float("inf")), -1), (dict(window=-1), -1),
                     (dict(sink=-1), -1), (dict(q=0), -1), (dict(q=A + 4), -1), (dict(out=0), -1), (dict(lse=0), -1), (dict(lse=A + 2), -1), (dict(status=A + 1), -1),
                     (dict(q_stride_t=63), -1), (dict(o_stride_h=60), -1), (dict(out=A + 64), -1), (dict(hq=2 ** 31 - 2, out=1 << 62), -4)):
        assert go(_ref(c), ctypes.byref(_attn(**kw)), A, 6, A, 1 << 40, None) == want, kw
    ok = ctypes.byref(_attn())
    assert go(_ref(c), None, A, 6, A, need, None) == -1
    assert go(_ref(c), ok, None, 6, A, need, None) == -1
    assert go(_ref(c), ok, A + 2, 6, A, need, None) == -1
    assert go(_ref(c), ok, A, -1, A, need, None) == -1
    assert go(_ref(c), ok, A, (1 << 25) + 1, A, 1 << 40, None) == -4
    assert go(_ref(c), ok, A, 6, None, need, None) == -5
    assert go(_ref(c), ok, A, 6, A, need - 1, None) == -5
    assert go(_ref(c), ok, A, 6, A + 128, need, None) == -5
    for other in (P.DCP_BF16, P.DCP_F32):
        assert go(_ref(_cache(dtype=other)), ok, A, 6, A, 1 << 40, None) == -4 and "dcp_block_attn_fwd" in P.dcp_last_error()
    full = _cache8(max_pages=1 << 26)   # 2^30 tokens a row
    assert go(_ref(full), ctypes.byref(_attn(n=16384, out=A << 20)), A, 16384, A, 1 << 40, None) == -4 and "2^31" in P.dcp_last_error()
    # nothing to do is legal
    assert go(_ref(c), ctypes.byref(_attn(n=0)), None, 6, None, 0, None) == 0
    assert go(_ref(c), ok, None, 0, None, 0, None) == 0


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_cache_host_code_under_address_and_ub_sanitizers(tmp_path):
    """cache_api.hip, cache_read_api.hip and paged_chunk_api.hip against host walks of the kernels: fake_cache.cpp, with those that know 8 bits in fake_cache8.cpp."""
    srcs = [(os.path.join(CSRC, f), []) for f in ("plan.cpp", "api.hip", "executor.hip", "cache_api.hip", "cache_read_api.hip", "paged_chunk_api.hip")] + \
           [(os.path.join(HERE, "fake_device.cpp"), []), (os.path.join(HERE, "fake_cache.cpp"), ["-Dlaunch_paged_attn=launch_paged_attn_other", "-Dlaunch_append=launch_append_other"]),
            (os.path.join(HERE, "fake_cache8.cpp"), []), (os.path.join(HERE, "cache8_driver.cpp"), [])]

    def compile_one(x):
        src, more = x
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        r = subprocess.run(["g++", "-x", "c++"] + FLAGS + more + ["-c", src, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        return obj
    with ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(compile_one, srcs))
    exe = str(tmp_path / "host_asan_cache8")
    r = subprocess.run(["g++", "-fsanitize=address,undefined"] + objs + ["-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe, "80"], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and "host-asan cache8 ok" in r.stdout, (r.stdout[-3000:] + r.stderr[-6000:])
