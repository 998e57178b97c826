"""Arithmetic of the calls on a paged cache at the limits that the host accepts, on the CPU under the undefined-behaviour sanitizer."""
import os
import shutil
import subprocess

import pytest

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


pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


def test_sums_of_needs_up_to_the_most_pages(tmp_path):
    _run(tmp_path, "sums")
