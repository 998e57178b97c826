"""dcp_cache_append in 8 bits for places that begin below row 0 of the new tokens or end behind them: the host's code and the index arithmetic of its kernel under
sanitizers, in tests/host_asan/append8_begins.cpp.  No GPU, no HIP runtime: g++ only."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_host_asan import CSRC, FLAGS, HERE


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_append_of_places_that_begin_below_row_0(tmp_path):
    srcs = [(os.path.join(CSRC, f), []) for f in ("plan.cpp", "api.hip", "executor.hip", "cache_api.hip")] + \
           [(os.path.join(HERE, "fake_device.cpp"), []), (os.path.join(HERE, "fake_cache.cpp"), ["-Dlaunch_paged_attn=launch_paged_attn_other", "-Dlaunch_append=launch_append_other"]),
            (os.path.join(HERE, "fake_cache8.cpp"), ["-Dlaunch_append=launch_append_8"]), (os.path.join(HERE, "append8_begins.cpp"), [])]

    def compile_one(x):
        src, more = x
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        r = subprocess.run(["g++", "-x", "c++"] + FLAGS + more + ["-c", src, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        return obj
    with ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(compile_one, srcs))
    exe = str(tmp_path / "host_asan_append8")
    r = subprocess.run(["g++", "-fsanitize=address,undefined"] + objs + ["-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and "host-asan append8 ok" in r.stdout, (r.stdout[-3000:] + r.stderr[-6000:])
