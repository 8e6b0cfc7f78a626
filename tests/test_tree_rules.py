"""Where the bits of a drafted tree are read, on the CPU: tests/host_rules/tree_rules.hip,
compiled for the host only (it calls no HIP function) with undefined behaviour trapped."""
import os
import subprocess

from paper_2505_08098_amd import build as lib_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rules(tmp_path):
    exe = tmp_path / "tree_rules"
    subprocess.run([lib_build.hipcc(), "-O1", "-std=c++17", "-Wall", "--offload-host-only",
                    "-Xarch_host", "-fsanitize=undefined",
                    "-Xarch_host", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2505_08098_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host_rules", "tree_rules.hip"),
                    "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    assert res.stdout.strip() == "ok"
