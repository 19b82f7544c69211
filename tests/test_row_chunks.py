"""Host check of the chunks that the layer norm's launches cut rows into: compiles tests/row_chunks_check.cpp against
the kernels' internal header and runs it on the CPU."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_32415_amd", "csrc")


def test_chunks_cover_the_rows(tmp_path):
    cc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(cc):
        pytest.skip("hipcc not found")
    exe = str(tmp_path / "row_chunks_check")
    src = os.path.join(ROOT, "tests", "row_chunks_check.cpp")
    r = subprocess.run([cc, "-x", "hip", "--offload-arch=gfx950", "-O2", "-std=c++17", "-Xarch_host",
                        "-fsanitize=signed-integer-overflow", "-Xarch_host", "-fno-sanitize-recover=all", "-I", CSRC,
                        src, "-o", exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "violations 0" in r.stdout
