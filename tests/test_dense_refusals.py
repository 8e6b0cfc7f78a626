"""What the dense operators refuse, through the C ABI and the binding, on the CPU:
every refusal comes before any device work."""
import ctypes
import math
import time

import numpy as np
import pytest
import torch

from paper_2505_08098_amd import dense

OK, INVALID, UNSUPPORTED, HIP, TOO_LARGE = 0, 1, 3, 5, 6
F16, BF16, F32, FP8 = 0, 1, 2, 3
A = 1 << 20  # an address that is never read

pytestmark = pytest.mark.skipif(torch.cuda.is_available(),
                                reason="made-up addresses: only where nothing can launch")


@pytest.fixture(scope="module")
def lib():
    return dense._lib()


def _ints(x):
    return None if x is None else np.asarray(x, dtype=np.int32)


def _plan(lib, q, k, ql=None, kl=None, n=None, heads=4, kv=2, d=64):
    arrays = [_ints(x) for x in (q, k, ql, kl)]
    ptr = [None if a is None else a.ctypes.data for a in arrays]
    n = (len(q) if q is not None else len(k)) - 1 if n is None else n
    h = lib.f3s_cross_plan(*ptr, n, heads, kv, d)
    assert not h  # (no device here)
    return lib.f3s_last_error()


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(n=-1), INVALID),
    (dict(heads=3), INVALID), (dict(heads=0), INVALID), (dict(kv=0), INVALID),
    (dict(kv=-2), INVALID),
    (dict(d=0), UNSUPPORTED), (dict(d=48), UNSUPPORTED), (dict(d=288), UNSUPPORTED),
    (dict(d=-64), UNSUPPORTED), (dict(heads=131072, kv=2), UNSUPPORTED),
    (dict(q=[1, 3, 9]), INVALID), (dict(k=[2, 3, 9]), INVALID),
    (dict(q=[0, 9, 3]), INVALID), (dict(k=[0, 9, 3]), INVALID),
    (dict(ql=[3, 7]), INVALID), (dict(ql=[-1, 3]), INVALID),
    (dict(kl=[5, 5]), INVALID), (dict(kl=[0, -4]), INVALID),
    (dict(q=[0, 3, 2147483647]), TOO_LARGE), (dict(k=[0, 3, 2147483647]), TOO_LARGE),
    (dict(), HIP),
])
def test_cross_plan(lib, change, status):
    args = dict(q=[0, 3, 9], k=[0, 4, 10])
    args.update(change)
    assert _plan(lib, **args) == status


def test_cross_calls_without_a_plan(lib):
    assert lib.f3s_cross_forward_workspace_bytes(None) == 0
    assert lib.f3s_cross_backward_workspace_bytes(None) == 0
    lib.f3s_cross_destroy(None)
    assert lib.f3s_cross_forward(None, A, A, A, F16, A, A, 1.0, None, 0, None) == INVALID
    assert lib.f3s_cross_backward(None, A, A, A, F16, A, A, A, A, A, A, 1.0, None, 0,
                                  None) == INVALID
    assert lib.f3s_last_error() == INVALID


def _cache(**change):
    f = dict(k=A, v=2 * A, k_exp=3 * A, v_exp=4 * A, n_pages=8, n_kv_heads=2, page_size=16,
             d=64)
    f.update(change)
    return dense._CacheStruct(*(f[n] for n, _ in dense._CacheStruct._fields_))


BAD_CACHES = [
    (dict(d=0), UNSUPPORTED), (dict(d=40), UNSUPPORTED), (dict(d=512), UNSUPPORTED),
    (dict(page_size=0), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED),
    (dict(page_size=24), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED),
    (dict(page_size=-16), UNSUPPORTED),
    (dict(n_pages=0), INVALID), (dict(n_kv_heads=0), INVALID),
    (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(k_exp=0), INVALID),
    (dict(v_exp=0), INVALID), (dict(k=A + 8), INVALID), (dict(v_exp=A + 4), INVALID),
]


def _write(lib, cache, K=5 * A, V=6 * A, dtype=F16, table=7 * A, pages=4, lens=8 * A, B=3, n=2):
    return lib.f3s_cache_write(ctypes.byref(cache) if cache else None, K, V, dtype, table,
                               pages, lens, B, n, None)


def _read(lib, cache, K=5 * A, V=6 * A, dtype=F16, table=7 * A, pages=4, lens=8 * A, B=3, n=2):
    return lib.f3s_cache_read(ctypes.byref(cache) if cache else None, K, V, dtype, table,
                              pages, lens, B, n, None)


def _attend(lib, cache, Q=16 * A, dtype=F16, O=17 * A, lse=18 * A, table=7 * A, pages=400,
            lens=8 * A, B=3, n=2, heads=4, prefix=None, P=0, scale=0.1, ws=32 * A,
            nbytes=1 << 40):
    return lib.f3s_cache_attend(ctypes.byref(cache) if cache else None, Q, dtype, O, lse,
                                table, pages, lens, B, n, heads, prefix, P, scale, ws, nbytes,
                                None)


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches(lib, change, status):
    c = _cache(**change)
    for call in (_write, _read, _attend):
        assert call(lib, c) == status and lib.f3s_last_error() == status
    for call in (_write, _read, _attend):
        assert call(lib, None) == INVALID


@pytest.mark.parametrize("call", [_write, _read])
@pytest.mark.parametrize("change,status", [
    (dict(B=-1), INVALID), (dict(n=-1), INVALID), (dict(pages=-1), INVALID),
    (dict(lens=None), INVALID), (dict(lens=8 * A + 2), INVALID), (dict(table=None), INVALID),
    (dict(table=7 * A + 1), INVALID), (dict(dtype=FP8), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED),
    (dict(K=5 * A + 8), INVALID), (dict(V=6 * A + 2), INVALID),
    (dict(K=A), INVALID), (dict(V=4 * A), INVALID), (dict(K=2 * A - 16), INVALID),  # the cache
    (dict(B=1 << 20, n=1 << 11), TOO_LARGE), (dict(B=1 << 19, n=1 << 10), TOO_LARGE),
    (dict(B=0), OK), (dict(n=0), OK), (dict(B=0, lens=None, table=None), OK),
    (dict(), HIP),
])
def test_write_and_read(lib, call, change, status):
    assert call(lib, _cache(), **change) == status


def test_write_takes_no_null_rows_and_no_fp32(lib):
    assert _write(lib, _cache(), K=None) == INVALID
    assert _write(lib, _cache(), V=None) == INVALID
    assert _write(lib, _cache(), dtype=F32) == UNSUPPORTED
    assert _read(lib, _cache(), K=None, V=None) == OK
    assert _read(lib, _cache(), dtype=F32) == HIP
    assert _read(lib, _cache(), K=7 * A) == INVALID and _read(lib, _cache(), V=8 * A) == INVALID
    assert _read(lib, _cache(), V=5 * A + 64) == INVALID     # K
    assert _write(lib, _cache(), V=5 * A) == HIP             # the same rows as K and V


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), INVALID), (dict(n=-1), INVALID), (dict(pages=-1), INVALID),
    (dict(heads=3), INVALID), (dict(heads=0), INVALID), (dict(heads=-4), INVALID),
    (dict(P=-1), INVALID), (dict(P=5), INVALID),
    (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
    (dict(dtype=F32), UNSUPPORTED), (dict(dtype=FP8), UNSUPPORTED),
    (dict(Q=None), INVALID), (dict(O=None), INVALID), (dict(lse=None), INVALID),
    (dict(lens=None), INVALID), (dict(table=None), INVALID),
    (dict(Q=16 * A + 4), INVALID), (dict(O=17 * A + 8), INVALID), (dict(lse=18 * A + 2), INVALID),
    (dict(prefix=9 * A + 2, P=5), INVALID),
    (dict(O=16 * A), INVALID),                       # onto Q
    (dict(O=A), INVALID), (dict(O=2 * A + 64), INVALID),   # onto the codes
    (dict(lse=3 * A), INVALID), (dict(lse=7 * A), INVALID), (dict(lse=8 * A), INVALID),
    (dict(lse=17 * A), INVALID), (dict(O=32 * A), INVALID),
    (dict(ws=None), INVALID), (dict(ws=32 * A + 16), INVALID), (dict(nbytes=4096), INVALID),
    (dict(B=1 << 20, n=1 << 11), TOO_LARGE), (dict(pages=1 << 28), TOO_LARGE),
    (dict(B=1 << 17, n=1 << 8), TOO_LARGE),
    (dict(prefix=9 * A, P=(1 << 30) + 1), TOO_LARGE),
    (dict(B=(1 << 31) - 1, n=(1 << 31) - 1, heads=1 << 30), TOO_LARGE),
    (dict(B=0), OK), (dict(n=0), OK),
    (dict(), HIP), (dict(prefix=9 * A, P=5), HIP),
    (dict(pages=16, ws=None, nbytes=0), HIP),        # short tables need no workspace
])
def test_attend(lib, change, status):
    assert _attend(lib, _cache(), **change) == status


def test_attend_workspace(lib):
    c = _cache()
    size = lambda *a: lib.f3s_cache_attend_workspace_bytes(ctypes.byref(c), *a)
    assert size(56, 3, 1, 4, 0) == 0            # 896 keys: one workgroup has them all
    assert size(57, 3, 1, 4, 0) > 0
    assert size(16, 3, 1, 4, 1) > 0
    assert size(400, 3, 2, 4, 100) <= size(400, 3, 2, 4, 100000)
    assert size(400, 3, 2, 3, 0) == 0 and size(-1, 3, 2, 4, 0) == 0
    assert size(400, 0, 2, 4, 0) == 0 and size(400, 3, 2, 4, -1) == 0
    assert lib.f3s_cache_attend_workspace_bytes(None, 4, 3, 1, 4, 0) == 0
    # what is asked for is enough, and a byte less is not
    n = size(400, 3, 2, 4, 100)
    assert _attend(lib, c, prefix=9 * A, P=100, nbytes=n) == HIP
    # (the rule takes the kernel of few rows here, which needs all of it)
    assert n % 256 == 0


# ---- the binding ------------------------------------------------------------------

@pytest.mark.parametrize("q,k,kw", [
    ([0.0, 2.0], [0, 2], {}), ([[0, 2]], [0, 2], {}), ([], [0], {}), ([0, 2], [0, 1, 2], {}),
    ([0, -2], [0, 2], {}), ([0, 2**31], [0, 2], {}), ([0, 2], [0, 2], dict(q_len=[1, 1])),
    ([0, 2], [0, 2], dict(k_len=[])), ([0, 2], [0, 2], dict(q_len=[0.5])),
    ([0, 2], [0, 2], dict(device="cpu")),
])
def test_plan_arguments(q, k, kw):
    with pytest.raises(ValueError):
        dense.CrossPlan(q, k, 4, 2, 64, **kw)


def test_cache_arguments():
    t = torch.zeros((2, 2, 16, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    e = torch.zeros((2, 2, 16), dtype=torch.uint8)
    with pytest.raises(TypeError):
        dense.Cache(t, t, e, e)                 # not on a GPU
    with pytest.raises(ValueError):
        dense.Cache(e, e, e, e)
    with pytest.raises(ValueError):
        dense.Cache([1], t, e, e)


@pytest.mark.parametrize("q_ptr, k_ptr, heads, kv", [
    ([0, 1], [0, 2**31 - 1], 65535, 65535),        # 2^37 keys of all heads
    ([0, 2**31 - 1], [0, 1], 1000, 1000),          # 2^31 rows of many heads
    (range(40001), range(40001), 8000, 8000),      # a tile for each of 3.2e8 rows
])
def test_plans_of_too_many_tiles_are_refused_at_once(lib, q_ptr, k_ptr, heads, kv):
    """Before lists of them are made, which memory would not hold."""
    start = time.monotonic()
    assert _plan(lib, q_ptr, k_ptr, heads=heads, kv=kv, d=32) == TOO_LARGE
    assert time.monotonic() - start < 10


def test_a_plan_of_many_sequences_is_divided_soon(lib):
    """200,000 sequences, one with a million keys: without a GPU the plan then
    fails, for want of one."""
    n = 200000
    k = [0] + [10**6 + 100 * b for b in range(n)]
    start = time.monotonic()
    assert _plan(lib, range(n + 1), k, heads=4, kv=1) == HIP
    assert time.monotonic() - start < 10
