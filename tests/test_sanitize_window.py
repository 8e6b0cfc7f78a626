"""The host code of windows, trees, accepted tokens and pages under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only, no GPU needed), driven through the C ABI by
tests/sanitize/window_sanitize.c."""
import concurrent.futures
import glob
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
       "-Xarch_host", "-fno-omit-frame-pointer"]


def test_window_host_code_under_asan_and_ubsan(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2505_08098_amd import build as lib_build
    hipcc = lib_build.hipcc()
    clang = os.path.join(ROCM, "llvm", "bin", "clang")
    rt = glob.glob(os.path.join(ROCM, "llvm", "lib", "clang", "*", "lib", "linux",
                                "libclang_rt.asan-x86_64.so"))
    if not os.path.exists(clang) or not rt or shutil.which(hipcc) is None and \
            not os.path.exists(hipcc):
        pytest.skip("ROCm clang with the ASan runtime is not available")
    csrc = os.path.join(ROOT, "paper_2505_08098_amd", "csrc")
    inc = ["-I", os.path.join(ROOT, "include"), "-I", csrc]
    # every source: the entry points share files with the others' checks
    cmds = [[hipcc, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *SAN, *inc,
             "-c", os.path.join(csrc, s), "-o", str(tmp_path / s.replace(".hip", ".o"))]
            for s in lib_build.SOURCES]
    with concurrent.futures.ThreadPoolExecutor(min(8, len(cmds))) as pool:
        for cmd, res in zip(cmds, pool.map(
                lambda c: subprocess.run(c, capture_output=True, text=True), cmds)):
            assert res.returncode == 0, res.stderr[-2000:]
    lib = tmp_path / "libf3s_san.so"
    subprocess.run([os.path.join(ROCM, "llvm", "bin", "clang++"), "-shared", "-fPIC",
                    "-fsanitize=address,undefined", "-shared-libasan", "-o", str(lib),
                    *[c[-1] for c in cmds], "-L", os.path.join(ROCM, "lib"), "-lamdhip64"],
                   check=True)
    exe = tmp_path / "window_sanitize"
    subprocess.run([clang, "-std=c11", "-g", "-fsanitize=address,undefined", "-shared-libasan",
                    "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__", *inc, "-I",
                    os.path.join(ROCM, "include"),
                    os.path.join(ROOT, "tests", "sanitize", "window_sanitize.c"), "-o",
                    str(exe), "-L", str(tmp_path), "-lf3s_san", "-L",
                    os.path.join(ROCM, "lib"), "-lamdhip64", "-lm",
                    "-Wl,-rpath," + str(tmp_path), "-Wl,-rpath," + os.path.join(ROCM, "lib"),
                    "-Wl,-rpath," + os.path.dirname(rt[0])], check=True)
    # leaks inside the (uninstrumented) HIP runtime are not the library's
    supp = tmp_path / "lsan.supp"
    supp.write_text("leak:libamdhip64\nleak:libhsa-runtime64\nleak:libamd_comgr\n"
                    "leak:libdrm\nleak:libnuma\n")
    env = dict(os.environ,
               ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0",
               LSAN_OPTIONS=f"suppressions={supp}",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1",
               HIP_VISIBLE_DEVICES="-1")
    res = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr[-4000:]
    assert res.stdout.strip() == "ok"
