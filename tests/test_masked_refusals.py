"""What attention over the cache with a window or a tree refuses, through the C ABI, on
the CPU: every refusal comes before any device work."""
import ctypes
import math

import pytest
import torch

from paper_2505_08098_amd import dense
from test_dense_refusals import (A, BAD_CACHES, F32, FP8, HIP, INVALID, OK, TOO_LARGE, UNSUPPORTED,
                                 _cache)

pytestmark = pytest.mark.skipif(torch.cuda.is_available(),
                                reason="made-up addresses: only where nothing can launch")


def _window(cache, Q=16 * A, dtype=0, O=17 * A, lse=18 * A, table=7 * A, pages=400, lens=8 * A,
            B=3, n=2, heads=4, window=5000, sinks=4, scale=0.1, ws=32 * A, nbytes=1 << 40):
    return dense._lib().f3s_cache_attend_window(
        ctypes.byref(cache) if cache else None, Q, dtype, O, lse, table, pages, lens, B, n, heads,
        window, sinks, scale, ws, nbytes, None)


def _tree(cache, Q=16 * A, dtype=0, O=17 * A, lse=18 * A, table=7 * A, pages=400, lens=8 * A,
          B=3, n=2, heads=4, parents=10 * A, prefix=None, P=0, scale=0.1, ws=32 * A,
          nbytes=1 << 40):
    return dense._lib().f3s_cache_attend_tree(
        ctypes.byref(cache) if cache else None, Q, dtype, O, lse, table, pages, lens, B, n, heads,
        parents, prefix, P, scale, ws, nbytes, None)


BOTH = [
    (dict(B=-1), INVALID), (dict(n=-1), INVALID), (dict(pages=-1), INVALID),
    (dict(heads=3), INVALID), (dict(heads=0), INVALID),
    (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
    (dict(dtype=F32), UNSUPPORTED), (dict(dtype=FP8), UNSUPPORTED),
    (dict(Q=None), INVALID), (dict(O=None), INVALID), (dict(lse=None), INVALID),
    (dict(lens=None), INVALID), (dict(table=None), INVALID),
    (dict(Q=16 * A + 4), INVALID), (dict(O=17 * A + 8), INVALID), (dict(lse=18 * A + 2), INVALID),
    (dict(O=16 * A), INVALID), (dict(O=A), INVALID), (dict(lse=3 * A), INVALID),
    (dict(lse=7 * A), INVALID), (dict(lse=8 * A), INVALID), (dict(lse=17 * A), INVALID),
    (dict(O=32 * A), INVALID), (dict(Q=32 * A + 256), INVALID), (dict(lens=32 * A + 512), INVALID),
    (dict(ws=None), INVALID), (dict(ws=32 * A + 16), INVALID), (dict(nbytes=4096), INVALID),
    (dict(pages=1 << 28), TOO_LARGE), (dict(B=1 << 24, n=200), TOO_LARGE),
    (dict(B=0), OK), (dict(n=0), OK), (dict(), HIP), (dict(n=200), HIP),
    (dict(pages=16, ws=None, nbytes=0), HIP),        # short tables need no workspace
]


@pytest.mark.parametrize("call", [_window, _tree])
@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches(call, change, status):
    assert call(_cache(**change)) == status and dense._lib().f3s_last_error() == status
    assert call(None) == INVALID


@pytest.mark.parametrize("call", [_window, _tree])
@pytest.mark.parametrize("change,status", BOTH)
def test_both(call, change, status):
    assert call(_cache(), **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(window=0, sinks=0), HIP),
    (dict(window=2**31 - 1, sinks=2**31 - 1), HIP),
    (dict(window=500, ws=None, nbytes=0), HIP),      # a short window needs no workspace
    (dict(n=1000, B=1, window=10), HIP),
])
def test_window(change, status):
    assert _window(_cache(), **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(parents=None), INVALID), (dict(parents=10 * A + 2), INVALID),
    (dict(parents=17 * A), INVALID), (dict(parents=32 * A + 300), INVALID),
    (dict(parents=18 * A), INVALID), (dict(parents=None, n=0), OK),
    (dict(n=256), HIP), (dict(n=257), UNSUPPORTED), (dict(n=257, B=0), UNSUPPORTED),
    (dict(P=-1), INVALID), (dict(P=5), INVALID), (dict(prefix=9 * A + 2, P=5), INVALID),
    (dict(prefix=9 * A, P=(1 << 30) + 1), TOO_LARGE), (dict(prefix=9 * A, P=5), HIP),
])
def test_tree(change, status):
    assert _tree(_cache(), **change) == status


def test_workspaces():
    c = _cache()
    L = dense._lib()
    window = lambda *a: L.f3s_cache_attend_window_workspace_bytes(ctypes.byref(c), *a)
    tree = lambda *a: L.f3s_cache_attend_tree_workspace_bytes(ctypes.byref(c), *a)
    for n in (1, 100):
        size = window(400, 3, n, 4, 5000, 4)
        assert size % 256 == 0 and size > 0
        assert _window(c, n=n, nbytes=size) == HIP and _window(c, n=n, nbytes=size - 1) == INVALID
        # no more than the window can need, however long the table
        assert window(1 << 20, 3, n, 4, 5000, 4) == window(1 << 24, 3, n, 4, 5000, 4)
        size = tree(400, 3, n, 4, 0)
        assert size > 0
        assert _tree(c, n=n, nbytes=size) == HIP and _tree(c, n=n, nbytes=size - 1) == INVALID
        assert tree(400, 3, n, 4, 100) >= tree(400, 3, n, 4, 0)
    for bad in ((400, 3, 2, 3, 5, 5), (-1, 3, 2, 4, 5, 5), (400, 0, 2, 4, 5, 5),
                (400, 3, 2, 4, -1, 5), (400, 3, 2, 4, 5, -1)):
        assert window(*bad) == 0
    for bad in ((400, 3, 2, 3, 0), (400, 3, 257, 4, 0), (400, 3, 2, 4, -1)):
        assert tree(*bad) == 0
    assert L.f3s_cache_attend_window_workspace_bytes(None, 4, 3, 1, 4, 9, 0) == 0
    assert L.f3s_cache_attend_tree_workspace_bytes(None, 4, 3, 1, 4, 0) == 0
