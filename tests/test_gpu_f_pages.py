"""Page tables and the moving of accepted tokens on the GPU against plain Python."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def assign(free, count, table, old, new, page, n):
    """The operator from its definition, on lists; free and table change."""
    n_pages, room = len(free), (len(table[0]) if table else 0) * page
    old, new = ([min(max(x, 0), room) for x in y] for y in (old, new))
    pages = lambda x: -(-x // page)
    count = min(max(count, 0), n_pages)
    for b, row in enumerate(table):
        for e in range(pages(new[b]), pages(old[b])):
            if 0 <= row[e] < n_pages and count < n_pages:
                free[count] = row[e]
                count += 1
            row[e] = -1
    need = sum(max(0, pages(y) - pages(x)) for x, y in zip(old, new))
    given = min(need, count)
    taken = free[count - given: count]
    got, slots = [], []
    for b, row in enumerate(table):
        have, want = pages(old[b]), pages(new[b])
        held = min(have, want)
        for e in range(have, want):
            row[e] = taken.pop(0) if taken else -1
            if row[e] != -1:
                held += 1
        got.append(min(new[b], held * page))
        for t in range(n):
            p = new[b] - n + t
            there = 0 <= p < got[b] and 0 <= row[p // page] < n_pages
            slots.append(row[p // page] * page + p % page if there else -1)
    return count - given, got, slots


def _check(gpu, gen, B, M, page, n, most, n_pages, steps=4):
    pool = gpu.PagePool.full(n_pages, page, device=DEV)
    order = torch.randperm(n_pages, generator=gen).to(torch.int32)
    pool.free.copy_(order)
    table = torch.full((B, M), -1, dtype=torch.int32, device=DEV)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    free, count, rows = order.tolist(), n_pages, table.tolist()
    for step in range(steps):
        new = torch.randint(0, most + 1, (B,), generator=gen, dtype=torch.int32)
        new[torch.rand(B, generator=gen) < 0.3] = 0
        keep = torch.rand(B, generator=gen) < 0.2
        new = torch.where(keep, lens.cpu(), new)
        old = lens.tolist()
        got, slots = gpu.pages_assign(pool, table, lens, new.to(DEV), n=n)
        count, want, places = assign(free, count, rows, old, new.tolist(), page, n)
        assert got.tolist() == want
        assert slots.dtype == torch.int64 and slots.flatten().tolist() == places
        assert table.tolist() == rows
        assert int(pool.count) == count and pool.free.tolist()[:count] == free[:count]
        # every page is in one place
        held = [e for b, row in enumerate(rows) for e in row[: -(-want[b] // page)]]
        assert sorted(held + free[:count]) == list(range(n_pages))
        lens = got
    return pool, table, lens


@pytest.mark.parametrize("B,M,page,n,most,n_pages", [
    (1, 4, 16, 1, 64, 4), (1, 1, 256, 3, 256, 1), (5, 7, 16, 20, 112, 40), (5, 7, 16, 0, 112, 9),
    (64, 20, 32, 5, 640, 700), (65, 100, 64, 2, 6400, 2000), (1000, 30, 16, 7, 480, 20000),
    (1024, 128, 16, 32, 2048, 60000),                     # the largest by one workgroup
    (1025, 20, 16, 3, 320, 9000), (3, 70000, 16, 1, 1120000, 150000),
    (40, 10, 16, 900, 160, 300), (2500, 3, 128, 1, 384, 5000),
    (16384, 2, 16, 1, 32, 20000), (20001, 2, 16, 1, 32, 30000),   # the last of three launches
])
def test_against_the_definition(gpu, B, M, page, n, most, n_pages):
    gen = torch.Generator().manual_seed(B + M)
    _check(gpu, gen, B, M, page, n, most, n_pages, steps=3 if B * M > 10000 else 6)


@pytest.mark.parametrize("B", [6, 1100])
def test_growing_and_shrinking_back_restores_the_pool(gpu, B):
    gen = torch.Generator().manual_seed(1)
    pool, table, lens = _check(gpu, gen, B, 40, 16, 4, 640, B * 15)
    before = [x.clone() for x in (pool.free, pool.count, table)]
    new = torch.randint(0, 641, (B,), generator=gen, dtype=torch.int32).to(DEV)
    held = int(pool.count)
    got, _ = gpu.pages_assign(pool, table, lens, new)
    back, _ = gpu.pages_assign(pool, table, got, lens)
    assert torch.equal(back, lens) and int(pool.count) == held
    assert torch.equal(pool.free[:held], before[0][:held])
    pages = -(-lens // 16)
    for b in range(B):
        assert torch.equal(table[b, : pages[b]], before[2][b, : pages[b]])


@pytest.mark.parametrize("B", [4, 1500])
def test_lengths_that_are_out_of_range_and_entries_that_are_no_pages(gpu, B):
    big = 2**31 - 1
    lens = [0, 40, -7, 48] * (B // 4)
    new = [big, -big, 20, 0] * (B // 4)
    n_pages = 3 * B
    rows = []
    for b in range(B):
        rows.append([[-1, -1, -1], [3 * b, 10**9, 3 * b + 1], [5, 5, 5], [-3, 3 * b, n_pages]][
            b % 4])
    table = _ints(rows)
    used = {p for b, row in enumerate(rows) if b % 4 in (1, 3) for p in row if 0 <= p < n_pages}
    free = [p for p in range(n_pages) if p not in used]
    count = len(free)
    free += [-1] * (n_pages - count)
    pool = gpu.PagePool(_ints(free), _ints([count]), 16)
    got, slots = gpu.pages_assign(pool, table, _ints(lens), _ints(new), n=3)
    count, want, places = assign(free, count, rows, lens, new, 16, 3)
    assert got.tolist() == want and slots.flatten().tolist() == places
    assert table.tolist() == rows
    assert int(pool.count) == count and pool.free.tolist()[:count] == free[:count]


@pytest.mark.parametrize("said", [-3, 2**31 - 1])
def test_a_count_out_of_range(gpu, said):
    pool = gpu.PagePool(_ints([4, 3, 2, 1, 0]), _ints([said]), 16)
    table = _ints([[-1, -1, -1]])
    got, _ = gpu.pages_assign(pool, table, _ints([0]), _ints([33]))
    if said < 0:
        assert got.tolist() == [0] and table.tolist() == [[-1, -1, -1]]
        assert int(pool.count) == 0
    else:
        assert got.tolist() == [33] and table.tolist() == [[2, 1, 0]]
        assert int(pool.count) == 2


def test_nothing_to_do(gpu):
    pool = gpu.PagePool.full(4, 16, device=DEV)
    got, slots = gpu.pages_assign(pool, torch.empty((0, 3), dtype=torch.int32, device=DEV),
                                  _ints([]), _ints([]), n=2)
    assert got.shape == (0,) and slots.shape == (0, 2)
    table = torch.empty((2, 0), dtype=torch.int32, device=DEV)
    got, slots = gpu.pages_assign(pool, table, _ints([0, 5]), _ints([3, 0]), n=2)
    assert got.tolist() == [0, 0] and (slots == -1).all() and int(pool.count) == 4


# ---- accepted tokens -----------------------------------------------------------------

def _full_cache(gpu, gen, n_pages, page, kv, d):
    codes = [torch.randint(0, 256, (n_pages, kv, page, d), generator=gen, dtype=torch.uint8)
             .to(DEV).view(torch.float8_e4m3fn) for _ in range(2)]
    powers = [torch.randint(0, 256, (n_pages, kv, page), generator=gen, dtype=torch.uint8)
              .to(DEV) for _ in range(2)]
    return gpu.Cache(*codes, *powers)


def _raw(cache):
    return [x.view(torch.uint8).cpu().clone() for x in (cache.k, cache.v, cache.k_exp,
                                                        cache.v_exp)]


def _keep(parts, table, lens, n, picks, page):
    """On host copies of the cache's parts; returns the new lengths."""
    n_pages, new = parts[0].shape[0], []
    for b, length in enumerate(lens):
        first = max(length, 0) - n
        front, kept, last = max(first, 0), 0, -1

        def place(p):
            e = p // page
            ok = e < len(table[b]) and 0 <= table[b][e] < n_pages
            return (table[b][e], p % page) if ok else None

        moves = []
        for t in picks[b]:
            if not (last < t < n and first + t >= 0):
                break
            moves.append((place(first + t), place(front + kept)))
            kept, last = kept + 1, t
        for x in parts:
            old = x.clone()
            for src, dst in moves:
                if src and dst:
                    x[dst[0], :, dst[1]] = old[src[0], :, src[1]]
        new.append(front + kept)
    return new


@pytest.mark.parametrize("d,kv,page,lens,n,picks", [
    (64, 2, 16, [40, 33, 17, 8], 8, [[0, 2, 5], [0, 1, 2], [7, -1, -1], [-1, 3, 4]]),
    (32, 1, 16, [20], 20, [list(range(1, 20)) + [-1]]),
    (128, 8, 64, [100, 64], 37, [[0, 36, -1], [3, 5, 4]]),           # not ascending: ends
    (96, 3, 32, [5, 3, 0, -4], 6, [[1, 3, 5], [0, 4, 5], [4, 5, -1], [0, 1, 2]]),  # padding
    (256, 2, 256, [600], 300, [list(range(0, 300, 2)) + [299, 300]]),
    (160, 5, 16, [900], 700, [list(range(3, 700, 2))]),              # more than one round
    (64, 40, 16, [30, 50], 12, [[1, 2, 9], [0, 0, 1]]),              # many heads
    (224, 1, 128, [130], 10, [[9]]), (192, 1, 16, [9], 5, [[]]),
])
def test_kept_rows_move(gpu, d, kv, page, lens, n, picks):
    gen = torch.Generator().manual_seed(d + n)
    B = len(lens)
    pages = -(-max(lens) // page)
    n_pages = B * pages + 2
    cache = _full_cache(gpu, gen, n_pages, page, kv, d)
    table = torch.randperm(n_pages, generator=gen)[: B * pages].view(B, pages).to(torch.int32)
    want = _raw(cache)
    new = gpu.cache_keep(cache, table.to(DEV), _ints(lens), n,
                         torch.tensor(picks, dtype=torch.int32, device=DEV).view(B, -1))
    lens_after = _keep(want, table.tolist(), lens, n, picks, page)
    assert new.tolist() == lens_after
    for a, b in zip(_raw(cache), want):
        assert torch.equal(a, b)


def test_kept_rows_without_places(gpu):
    """Rows whose page is none, before and after the move; lengths beyond the table."""
    gen = torch.Generator().manual_seed(3)
    cache = _full_cache(gpu, gen, 6, 16, 2, 64)
    table = [[0, -1, 1], [2, 99, 3], [4, 5, -1]]
    lens, n, picks = [45, 45, 70], 40, [[0, 12, 30, 39], [1, 11, 28, 38], [0, 1, 14, 39]]
    want = _raw(cache)
    new = gpu.cache_keep(cache, _ints(table), _ints(lens), n, _ints(picks))
    assert new.tolist() == _keep(want, table, lens, n, picks, 16)
    for a, b in zip(_raw(cache), want):
        assert torch.equal(a, b)


def test_a_draft_with_its_pages(gpu):
    """The operators together, as a step of generation uses them, captured: places for a
    draft, its rows written, what is accepted kept, the rest's pages given back."""
    B, n, page, kv, d, M = 5, 6, 16, 2, 64, 8
    pool = gpu.PagePool.full(B * M, page, device=DEV)
    cache = gpu.Cache.empty(B * M, page, kv, d, device=DEV)
    table = torch.full((B, M), -1, dtype=torch.int32, device=DEV)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    picks = torch.zeros((B, 3), dtype=torch.int32, device=DEV)
    K, V = (torch.zeros((B, n, kv, d), dtype=torch.float16, device=DEV) for _ in "KV")

    def step():
        got, slots = gpu.pages_assign(pool, table, lens, lens + n, n=n)
        gpu.cache_write(cache, K, V, table, got)
        kept = gpu.cache_keep(cache, table, got, n, picks)
        done, _ = gpu.pages_assign(pool, table, got, kept)
        lens.copy_(done)
        return slots

    def start():
        pool.free.copy_(torch.arange(B * M, dtype=torch.int32))
        pool.count.fill_(B * M)
        lens.zero_()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    start()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slots = step()
    start()
    gen = torch.Generator().manual_seed(4)
    rows = [[] for _ in range(B)]
    for turn in range(20):
        choice = [sorted(torch.randperm(n, generator=gen)[: int(torch.randint(
            0, 4, (1,), generator=gen))].tolist()) for _ in range(B)]
        # (multiples of 1/8 below 16: codes hold them)
        x = torch.randint(-15, 16, (B, n, kv, d), generator=gen).half()
        K.copy_(x)
        V.copy_(-x)
        picks.copy_(torch.tensor([c + [-1] * (3 - len(c)) for c in choice], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert bool((slots >= 0).all())
        for b in range(B):
            rows[b] += [x[b, t] for t in choice[b]]
        assert lens.tolist() == [len(r) for r in rows]
        held = sum(-(-len(r) // page) for r in rows)
        assert int(pool.count) == B * M - held
        longest = max(1, max(len(r) for r in rows))
        back, other = gpu.cache_read(cache, table, lens, longest)
        for b in range(B):
            m = len(rows[b])
            if m:
                assert torch.equal(back[b, longest - m:].cpu(), torch.stack(rows[b]))
                assert torch.equal(other[b, longest - m:].cpu(), -torch.stack(rows[b]))
        assert math.isfinite(float(back.float().abs().sum()))


def test_bad_arguments(gpu):
    pool = gpu.PagePool.full(8, 16, device=DEV)
    table, lens = _ints([[0, 1], [2, 3]]), _ints([1, 2])
    with pytest.raises(ValueError):
        gpu.pages_assign(pool, table, lens, _ints([1]))
    with pytest.raises(ValueError):
        gpu.pages_assign(pool, table, lens, lens, n=-1)
    with pytest.raises(TypeError):
        gpu.pages_assign(pool, table.long(), lens, lens)
    with pytest.raises(ValueError):
        gpu.pages_assign(pool, table, lens, lens, n=2**31)
    with pytest.raises(gpu.F3SError):
        gpu.pages_assign(gpu.PagePool.full(8, 24, device=DEV), table, lens, lens)
    with pytest.raises(gpu.F3SError):
        gpu.pages_assign(pool, pool.free[:4].view(2, 2), lens, lens)   # the pool as a table
    with pytest.raises(ValueError):
        gpu.PagePool(pool.free, pool.free, 16)
    cache = gpu.Cache.empty(8, 16, 1, 64, device=DEV)
    with pytest.raises(ValueError):
        gpu.cache_keep(cache, table, lens, 2, _ints([[0]]))
    with pytest.raises(TypeError):
        gpu.cache_keep(cache, table, lens, 2, torch.zeros((2, 1), device=DEV))
    with pytest.raises(gpu.F3SError):
        gpu.cache_keep(cache, table, lens, -1, _ints([[0], [0]]))
    one = gpu.Cache(cache.k, cache.k, cache.k_exp, cache.k_exp)
    with pytest.raises(gpu.F3SError):
        gpu.cache_keep(one, table, lens, 2, _ints([[0], [0]]))
