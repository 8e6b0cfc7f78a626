"""The rules of a window of keys on the CPU: tests/host_rules/window_rules.hip,
compiled for the host only (it calls no HIP function) with undefined behaviour
trapped; and what a window plan refuses, before any device work."""
import os
import subprocess
import time

import numpy as np
import pytest
import torch

from paper_2505_08098_amd import dense
from paper_2505_08098_amd import build as lib_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, HIP, TOO_LARGE = 1, 3, 5, 6
A = 1 << 20  # an address that is never read

no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                            reason="plans that only the lack of a GPU stops")


def test_rules(tmp_path):
    exe = tmp_path / "window_rules"
    subprocess.run([lib_build.hipcc(), "-O1", "-std=c++17", "-Wall", "--offload-host-only",
                    "-Xarch_host", "-fsanitize=undefined",
                    "-Xarch_host", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2505_08098_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host_rules", "window_rules.hip"),
                    "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    assert res.stdout.strip() == "ok"


def _plan(q, k, ql=None, kl=None, n=None, heads=4, kv=2, d=64, window=100, sinks=4):
    L = dense._lib()
    arrays = [None if x is None else np.asarray(x, dtype=np.int32) for x in (q, k, ql, kl)]
    ptr = [None if a is None else a.ctypes.data for a in arrays]
    n = (len(q) if q is not None else len(k)) - 1 if n is None else n
    h = L.f3s_window_plan(*ptr, n, heads, kv, d, window, sinks)
    assert not h  # (no device here)
    return L.f3s_last_error()


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(n=-1), INVALID),
    (dict(heads=3), INVALID), (dict(heads=0), INVALID), (dict(kv=0), INVALID),
    (dict(d=0), UNSUPPORTED), (dict(d=48), UNSUPPORTED), (dict(d=288), UNSUPPORTED),
    (dict(heads=131072, kv=2), UNSUPPORTED),
    (dict(window=-1), INVALID), (dict(sinks=-1), INVALID),
    (dict(q=[1, 3, 9]), INVALID), (dict(k=[2, 3, 9]), INVALID),
    (dict(q=[0, 9, 3]), INVALID), (dict(k=[0, 9, 3]), INVALID),
    (dict(ql=[3, 7]), INVALID), (dict(ql=[-1, 3]), INVALID),
    (dict(kl=[5, 5]), INVALID), (dict(kl=[0, -4]), INVALID),
    (dict(q=[0, 3, 2147483647]), TOO_LARGE), (dict(k=[0, 3, 2147483647]), TOO_LARGE),
    (dict(window=0, sinks=0), HIP), (dict(window=2**31 - 1, sinks=2**31 - 1), HIP),
    (dict(), HIP),
])
def test_plan(change, status):
    args = dict(q=[0, 3, 9], k=[0, 4, 10])
    args.update(change)
    assert _plan(**args) == status


def test_calls_without_a_plan():
    L = dense._lib()
    assert L.f3s_window_forward_workspace_bytes(None) == 0
    assert L.f3s_window_backward_workspace_bytes(None) == 0
    L.f3s_window_destroy(None)
    assert L.f3s_window_forward(None, A, A, A, 0, A, A, 1.0, None, 0, None) == INVALID
    assert L.f3s_window_backward(None, A, A, A, 0, A, A, A, A, A, A, 1.0, None, 0,
                                 None) == INVALID
    assert L.f3s_last_error() == INVALID


@no_gpu
@pytest.mark.parametrize("q, k, heads, kv, status", [
    ([0, 1], [0, 2**31 - 4097], 65535, 65535, TOO_LARGE),
    (range(40001), range(40001), 8000, 8000, TOO_LARGE),
    ([0, 300000], [0, 300000], 8, 8, HIP),
    (range(100001), [7 * b for b in range(100001)], 8, 2, HIP),
])
def test_large_plans_are_divided_or_refused_soon(q, k, heads, kv, status):
    start = time.monotonic()
    assert _plan(q, k, heads=heads, kv=kv, d=32) == status
    assert time.monotonic() - start < 10


@pytest.mark.parametrize("kw", [dict(window=-2**31), dict(window=2**31), dict(sinks=2**40),
                                dict(q_len=[1, 1]), dict(device="cpu"), dict(d=2**33)])
def test_plan_arguments(kw):
    with pytest.raises(ValueError):
        dense.WindowPlan([0, 2], [0, 2], 4, 2, **{"d": 64, **kw})
