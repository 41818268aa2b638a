"""Host logic of the linear-attention layer without a GPU, under AddressSanitizer and UndefinedBehaviorSanitizer:
linear.cpp and augtree.cpp are compiled with g++ together with CPU stand-ins for the HIP runtime and the kernel
launchers (tests/host/fake_hip.cpp, tests/host/linear_host_test.cpp), which check every launch's segments, blocks and
workspace arrays, the order of launches, and that a failing launch ends the call with AUGTREE_ERR_HIP."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33133_amd", "csrc")
HOST = os.path.join(ROOT, "tests", "host")


@pytest.mark.timeout(600)
def test_linear_host_logic_under_sanitizers(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir(HOST):
        pytest.skip("g++ or the host test sources not found")
    exe = str(tmp_path / "linear_host_test")
    # host-only build (no HIP source on this line): the sanitizers apply to host code
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-I" + HOST, os.path.join(CSRC, "augtree.cpp"),
           os.path.join(CSRC, "linear.cpp"), os.path.join(HOST, "fake_hip.cpp"),
           os.path.join(HOST, "linear_host_test.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=500)
    assert r.returncode == 0 and r.stdout.startswith("ok"), (r.stdout[-4000:] + r.stderr[-4000:])
    words = r.stdout.replace(",", "").split()
    assert int(words[3]) > 0 and int(words[5]) > 0, r.stdout  # tables and split scans were exercised
