"""Cached attention of very many sequences: each is one workgroup's, which finds it
by its number and not by looking through the lengths of all."""
import ctypes

import pytest
import torch

from paper_2505_08098_amd import dense
from test_dense_refusals import A


def _round256(n):
    return -(-n // 256) * 256


@pytest.mark.parametrize("B", [8193, 100000, 1 << 20])
def test_partial_results_are_one_per_row(B):
    """8 query heads over 2 key heads: no more partial rows than query rows."""
    c = dense._CacheStruct(A, 2 * A, 3 * A, 4 * A, 8, 2, 64, 64)
    rows = B * 8
    assert dense._lib().f3s_cache_attend_workspace_bytes(ctypes.byref(c), 100, B, 1, 8, 0) == \
        _round256(rows * 64 * 4) + _round256(rows * 8) + _round256(B * 8)


@pytest.mark.gpu
@pytest.mark.parametrize("room,P", [(64, 0), (3008, 0), (20000, 40)])
def test_many_sequences(gpu, room, P):
    from test_gpu_b_cache import DEV, _cache, _compare, _rows, _table
    gen = torch.Generator().manual_seed(room)
    kv, d, page, B = 2, 64, 16, 9000
    top = min(room, 15000)
    lens7 = [0, 1, min(63, top), 64, 17, 40, top]
    shared = -(-P // page)
    table7, n_pages = _table(gen, 7, -(-top // page), first=shared)
    cache = _cache(gpu, n_pages, page, kv, d)
    int32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    x = [_rows(gen, (7, top, kv, d), torch.float16).to(DEV) for _ in "KV"]
    gpu.cache_write(cache, *x, table7.to(DEV), int32([top] * 7))
    prefix, more = None, {}
    if P:
        prefix = torch.arange(shared, dtype=torch.int32)
        gpu.cache_write(cache, *(v[:1, :P].contiguous() for v in x), prefix.view(1, -1).to(DEV),
                        int32([P]))
        more = dict(prefix=prefix.to(DEV), prefix_len=P)
    Q7 = torch.randn((7, 1, 4, d), generator=gen).half()
    pick = torch.randint(0, 6, (B,), generator=gen)
    pick[[0, 4567, B - 1]] = 6                     # (three long ones)
    tables = torch.full((B, room // page), -1, dtype=torch.int32)
    tables[:, :table7.shape[1]] = table7[pick]
    lens = torch.tensor(lens7)[pick].to(torch.int32)
    O, lse = gpu.cache_attend(cache, Q7[pick].to(DEV), tables.to(DEV), lens.to(DEV), **more)
    first = [int((pick == k).nonzero()[0]) for k in range(7)]
    _compare(cache, Q7, table7, lens7, prefix, P, 0.125, O[first], lse[first])
    at = torch.tensor(first)[pick].to(DEV)
    assert torch.equal(O, O[at]) and torch.equal(lse, lse[at])
