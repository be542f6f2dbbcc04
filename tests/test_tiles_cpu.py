"""The bookkeeping of shared tiles (rv_tiles.h) and the entry points that use it
(rv_cache_ops.cpp) on the CPU, built with the address and undefined-behaviour
sanitizers: tests/host/tiles_check.cpp replaces device memory by host memory and
the kernels by plain loops.  Copies of every kind of move set, random walks of
copies, forks and writes against plain lists, attention plans, every refusal."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_moves_tables_plans_and_refusals(tmp_path):
    exe = str(tmp_path / "tiles_check")
    cmd = [HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-g", "-std=c++17", "-fno-gpu-sanitize",
           "-Xarch_host", "-fsanitize=address,undefined", "-Xarch_host", "-fno-sanitize-recover=all",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2505_18629_amd", "csrc"),
           os.path.join(ROOT, "tests", "host", "tiles_check.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-3000:]
    assert "as they should be" in r.stdout
