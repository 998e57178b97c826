"""The host code of the calls on a paged cache (csrc/cache_api.hip: checks, sizes of launches, workspaces) built for the CPU with
AddressSanitizer and UndefinedBehaviorSanitizer and driven through the C ABI by tests/host_asan/cache_driver.cpp, with the kernels
replaced by the host walks of tests/host_asan/fake_cache.cpp.  No GPU, no HIP runtime: g++ only."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_host_asan import CSRC, FLAGS, HERE


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_cache_host_code_under_address_and_ub_sanitizers(tmp_path):
    srcs = [os.path.join(CSRC, f) for f in ("plan.cpp", "api.hip", "executor.hip", "cache_api.hip")] + \
           [os.path.join(HERE, f) for f in ("fake_device.cpp", "fake_cache.cpp", "cache_driver.cpp")]

    def compile_one(src):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        r = subprocess.run(["g++", "-x", "c++"] + FLAGS + ["-c", src, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        return obj
    with ThreadPoolExecutor(max_workers=7) as ex:
        objs = list(ex.map(compile_one, srcs))
    exe = str(tmp_path / "host_asan_cache")
    r = subprocess.run(["g++", "-fsanitize=address,undefined"] + objs + ["-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe, "80"], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and "host-asan cache ok" in r.stdout, (r.stdout[-3000:] + r.stderr[-6000:])
