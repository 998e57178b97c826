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
