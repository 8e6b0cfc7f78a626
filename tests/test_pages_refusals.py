"""What the moving of accepted tokens and the page tables refuse, through the C ABI, on
the CPU: every refusal comes before any device work."""
import ctypes

import pytest
import torch

from paper_2505_08098_amd import dense
from test_dense_refusals import A, BAD_CACHES, HIP, INVALID, OK, TOO_LARGE, UNSUPPORTED, _cache

pytestmark = pytest.mark.skipif(torch.cuda.is_available(),
                                reason="made-up addresses: only where nothing can launch")


def _keep(cache, table=7 * A, pages=4, lens=8 * A, B=3, n=2, picks=9 * A, m=2, new=10 * A):
    return dense._lib().f3s_cache_keep(ctypes.byref(cache) if cache else None, table, pages,
                                       lens, B, n, picks, m, new, None)


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_keep_caches(change, status):
    assert _keep(_cache(**change)) == status and dense._lib().f3s_last_error() == status
    assert _keep(None) == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), INVALID), (dict(n=-1), INVALID), (dict(m=-1), INVALID), (dict(pages=-1), INVALID),
    (dict(lens=None), INVALID), (dict(table=None), INVALID), (dict(picks=None), INVALID),
    (dict(new=None), INVALID), (dict(lens=8 * A + 2), INVALID), (dict(table=7 * A + 1), INVALID),
    (dict(picks=9 * A + 3), INVALID), (dict(new=10 * A + 2), INVALID),
    (dict(new=8 * A), INVALID), (dict(new=7 * A + 44), INVALID), (dict(new=9 * A), INVALID),
    (dict(new=A), INVALID), (dict(lens=2 * A + 64), INVALID), (dict(table=3 * A), INVALID),
    (dict(picks=4 * A - 4), INVALID),
    (dict(B=0), OK), (dict(B=0, lens=None, new=None), OK),
    (dict(m=(1 << 30) + 1), TOO_LARGE), (dict(m=2**31 - 1), TOO_LARGE),
    (dict(m=0, picks=None), HIP), (dict(n=0), HIP), (dict(pages=0, table=None), HIP),
    (dict(new=7 * A + 48), HIP), (dict(), HIP),
])
def test_keep(change, status):
    assert _keep(_cache(), **change) == status


def test_keep_parts_that_share_memory():
    assert _keep(_cache(v=A, v_exp=3 * A)) == INVALID       # one place for keys and values
    assert _keep(_cache(v_exp=3 * A)) == INVALID
    assert _keep(_cache(k_exp=A)) == INVALID
    assert _keep(_cache(n_kv_heads=1 << 20), B=1 << 20) in (TOO_LARGE, INVALID)


def _assign(free=A, count=2 * A, n_pages=100, table=3 * A, pages=8, lens=4 * A, new=5 * A,
            got=6 * A, slots=7 * A, B=3, n=2, page=16, ws=8 * A, nbytes=1 << 30):
    return dense._lib().f3s_pages_assign(free, count, n_pages, table, pages, lens, new, got,
                                         slots, B, n, page, ws, nbytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(page=8), UNSUPPORTED), (dict(page=24), UNSUPPORTED), (dict(page=512), UNSUPPORTED),
    (dict(page=0), UNSUPPORTED), (dict(page=-16), UNSUPPORTED),
    (dict(n_pages=0), INVALID), (dict(pages=-1), INVALID), (dict(B=-1), INVALID),
    (dict(n=-1), INVALID),
    (dict(free=None), INVALID), (dict(count=None), INVALID), (dict(table=None), INVALID),
    (dict(lens=None), INVALID), (dict(new=None), INVALID), (dict(got=None), INVALID),
    (dict(slots=None), INVALID), (dict(free=A + 2), INVALID), (dict(slots=7 * A + 4), INVALID),
    (dict(table=3 * A + 2), INVALID), (dict(got=6 * A + 1), INVALID),
    (dict(got=4 * A), INVALID), (dict(got=5 * A + 8), INVALID), (dict(table=A + 396), INVALID),
    (dict(count=A), INVALID), (dict(slots=3 * A + 88), INVALID), (dict(slots=5 * A), INVALID),
    (dict(lens=A), INVALID),
    (dict(pages=1 << 26, page=32), TOO_LARGE), (dict(B=(1 << 24) + 1), TOO_LARGE),
    (dict(n=(1 << 30) + 1), TOO_LARGE), (dict(n=2**31 - 1, B=1), TOO_LARGE),
    (dict(B=0), OK), (dict(B=0, lens=None), OK),
    (dict(new=4 * A), HIP),                                  # the same lengths
    (dict(n=0, slots=None), HIP), (dict(ws=None, nbytes=0), HIP), (dict(), HIP),
    # larger batches need a workspace
    (dict(B=2000, ws=None), INVALID), (dict(B=2000, nbytes=64), INVALID),
    (dict(B=2000, ws=8 * A + 8), INVALID), (dict(B=2000, ws=4 * A), INVALID),
    (dict(B=2000, ws=3 * A), INVALID), (dict(B=2000), HIP),
])
def test_assign(change, status):
    assert _assign(**change) == status


def test_assign_workspace():
    size = dense._lib().f3s_pages_assign_workspace_bytes
    assert size(1024, 128, 32) == 0 and size(1, 1 << 17, 1) == 0
    for more in ((1025, 1, 1), (1024, 129, 1), (1024, 1, 33)):
        assert size(*more) > 4 * more[0]
        assert _assign(B=more[0], pages=more[1], n=more[2], nbytes=size(*more)) == HIP
        assert _assign(B=more[0], pages=more[1], n=more[2], nbytes=size(*more) - 1) == INVALID
    for bad in ((0, 5, 5), (-1, 5, 5), (5, -1, 5), (5, 5, -1), (2**31 - 1, 5, 5),
                (1, 5, (1 << 30) + 1)):
        assert size(*bad) == 0
