"""More of the paged KV cache's host logic without a GPU, under AddressSanitizer and UndefinedBehaviorSanitizer, on the
teams and stand-ins of tests/host/paged_host_test.cpp."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33133_amd", "csrc")
HOST = os.path.join(ROOT, "tests", "host")


@pytest.mark.timeout(600)
@pytest.mark.parametrize("name", ["paged_sums_test", "paged_lanes_test"])
def test_plans_under_sanitizers(tmp_path, name):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir(HOST):
        pytest.skip("g++ or the host test sources not found")
    exe = str(tmp_path / name)
    # host-only build (no HIP source on this line): the sanitizers apply to host code
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=undefined", "-pthread", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-I" + HOST, os.path.join(CSRC, "augtree.cpp"),
           os.path.join(CSRC, "paged.cpp"), os.path.join(HOST, "fake_hip.cpp"), os.path.join(HOST, name + ".cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=500)
    assert r.returncode == 0 and r.stdout.startswith("ok"), (r.stdout[-4000:] + r.stderr[-4000:])
