"""The paged cache's C entry points over a runtime that the test writes itself (paged_api_host.cpp)."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_attend_that_cannot_run_is_refused_alone(tmp_path):
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    out = str(tmp_path / "paged_api")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", include, os.path.join(HERE, "paged_api_host.cpp"), "-o", out])
    r = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout
