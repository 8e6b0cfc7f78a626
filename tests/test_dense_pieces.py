"""The smallest piece of a divided pass of cross attention, on the CPU:
tests/host_rules/dense_pieces.hip, compiled for the host only."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_dense_pieces(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2505_08098_amd import build as lib_build
    exe = tmp_path / "dense_pieces"
    subprocess.run([lib_build.hipcc(), "-O1", "-std=c++17", "-Wall", "--offload-host-only",
                    "-Xarch_host", "-fsanitize=undefined",
                    "-Xarch_host", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2505_08098_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host_rules", "dense_pieces.hip"),
                    "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout == "ok\n", res.stdout + res.stderr
