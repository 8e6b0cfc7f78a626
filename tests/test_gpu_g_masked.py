"""Attention over the 8-bit cache with a window or a tree of drafted tokens, on the GPU
against plain 64-bit attention: by the kernels of 16, 128 and 256 query rows."""
import math

import pytest
import torch

from _dense import attention, close, half_step
from test_gpu_b_cache import _cache, _rows, _table, _values

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
TYPES = [torch.float16, torch.bfloat16]


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def window_seen(lens, n, m, window, sinks):
    """[n, m]: the own positions that each of the n newest tokens sees."""
    p = max(lens, 0) - n + torch.arange(n)[:, None]
    j = torch.arange(m)
    return (j <= p) & ((p - j < window) | (j < sinks))


def tree_seen(lens, parents, m):
    n = len(parents)
    first = max(lens, 0) - n
    seen = torch.zeros((n, m), dtype=torch.bool)
    for t in range(n):
        if first + t < 0:
            continue
        seen[t, : max(0, min(first, m))] = True
        at = t
        while at >= 0:
            if 0 <= first + at < m:
                seen[t, first + at] = True
            at = parents[at] if 0 <= parents[at] < at else -1
    return seen


def _compare(cache, Q, table, lens, seen_of, scale, O, lse, prefix=None, prefix_len=0):
    """seen_of(b, m): [n, m] for sequence b with m keys."""
    dtype, page = Q.dtype, cache.page_size
    B, n, H, d = Q.shape
    g = H // cache.kv_heads
    values = _values(cache)

    def rows(pages, m):
        at = torch.arange(m)
        ok = (pages >= 0) & (pages < cache.n_pages)
        there = ok[at // page] if m else torch.zeros(0, dtype=torch.bool)
        k = pages[at // page].long().clamp(0, cache.n_pages - 1) if m else at
        return [torch.where(there[:, None, None], x[k, :, at % page], 0.0)
                for x in values] + [there]

    front = rows(prefix.cpu(), prefix_len) if prefix_len else None
    for b in range(B):
        m = min(max(lens[b], 0), table.shape[1] * page)
        k, v, there = rows(table[b], m)
        seen = seen_of(b, m) & there
        if front:
            k, v = (torch.cat([x, y]) for x, y in zip(front[:2], (k, v)))
            seen = torch.cat([front[2].expand(n, -1), seen], 1)
        for h in range(H):
            V = v[:, h // g]
            f = attention(Q[b, :, h].double(), k[:, h // g], V, scale, half_step(dtype),
                          up=2.0 ** -11, seen=seen)
            # a probability below f16's smallest, next to the largest power that the row
            # sees: half a step of 2^-24 of each key, times two for powers up to 2^-8 of it
            top = torch.where(seen, V.abs().amax(1), 0.0).amax(1) if m + prefix_len \
                else torch.zeros(n, dtype=torch.float64)
            tol = f["O_tol"] + (2.0 ** -24 * top * seen.sum(1))[:, None]
            what = (b, h, lens[b])
            close(O[b, :, h], f["O"], tol, ("O",) + what)
            close(lse[b, :, h], f["lse"], f["lse_tol"], ("lse",) + what)


def _setup(gpu, dtype, d, page, kv, g, lens, n, prefix_len=0, room=0, seed=0, spread=0):
    gen = torch.Generator().manual_seed(seed + d + page + n)
    B = len(lens)
    shared = -(-prefix_len // page)
    table, n_pages = _table(gen, B, max(1, -(-max(max(lens), room) // page)), first=shared)
    cache = _cache(gpu, n_pages, page, kv, d)
    lens_d = _ints(lens)
    prefix = None

    def states(shape):
        K, V = (_rows(gen, shape, dtype) for _ in "KV")
        if spread:  # values of very different sizes, a row each
            V = (V.double() * 2.0 ** torch.randint(-spread, spread + 1, shape[:3] + (1,),
                                                   generator=gen)).to(dtype)
        return K.to(DEV), V.to(DEV)

    if prefix_len:
        prefix = torch.arange(shared - 1, -1, -1, dtype=torch.int32, device=DEV)
        gpu.cache_write(cache, *states((1, prefix_len, kv, d)), prefix.view(1, -1),
                        _ints([prefix_len]))
    if max(lens) > 0:
        gpu.cache_write(cache, *states((B, max(lens), kv, d)), table.to(DEV), lens_d)
    Q = torch.randn((B, n, kv * g, d), generator=gen, dtype=torch.float64).to(dtype)
    return cache, Q, table, lens_d, prefix, gen


def _window_case(gpu, dtype, d, page, kv, g, lens, n, window, sinks, scale=None, **kw):
    cache, Q, table, lens_d, _, _ = _setup(gpu, dtype, d, page, kv, g, lens, n, **kw)
    scale = 1 / math.sqrt(d) if scale is None else scale
    O, lse = gpu.cache_attend_window(cache, Q.to(DEV), table.to(DEV), lens_d, window, sinks,
                                     scale=scale)
    torch.cuda.synchronize()
    _compare(cache, Q, table, lens, lambda b, m: window_seen(lens[b], n, m, window, sinks), scale,
             O, lse)


WINDOWS = [
    # d, page, key heads, query heads of each, lengths, new tokens, window, sinks
    (64, 16, 2, 1, [1, 0, 5, 33, 16, 17], 1, 8, 0),
    (64, 16, 1, 4, [300, 1, 64, 65], 1, 40, 3),
    (128, 64, 2, 4, [1000, 3, 517], 1, 100, 70),
    (32, 16, 3, 1, [40, 41, 3], 5, 7, 1),
    (96, 16, 1, 2, [290], 3, 1, 0), (64, 16, 1, 2, [290, 4], 3, 0, 5),
    (64, 16, 1, 2, [90], 3, 0, 0),
    (256, 256, 1, 3, [600, 20], 2, 128, 4),
    (160, 128, 1, 1, [129], 1, 2**31 - 1, 9), (192, 64, 1, 2, [64], 4, 17, 17),
    (224, 16, 1, 1, [15], 1, 3, 2**31 - 1),
    (64, 16, 1, 40, [70, 200], 1, 33, 2),
    # many rows
    (64, 16, 2, 2, [100, 130, 7, 0], 50, 20, 3),
    (64, 32, 1, 1, [300, 140], 140, 64, 0),
    (128, 64, 1, 4, [700, 333], 60, 100, 5),
    (128, 16, 1, 5, [500], 100, 2**31 - 1, 0), (32, 16, 2, 1, [400], 129, 31, 130),
    (96, 16, 1, 3, [200, 50], 66, 40, 66), (256, 128, 1, 2, [400], 70, 90, 2),
    (160, 32, 1, 2, [300], 40, 16, 0), (192, 16, 1, 3, [250], 31, 1, 7),
    (224, 64, 1, 2, [280, 40], 50, 55, 55), (64, 16, 1, 2, [140, 60], 80, 0, 9),
    (64, 16, 1, 2, [140], 80, 0, 0),
]


ROWS = ["16", "128", "256"]  # (256: d = 96 and 128 only, else by the rule)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("room", [0, 3000])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,page,kv,g,lens,n,window,sinks", WINDOWS)
def test_window(gpu, monkeypatch, rows, dtype, d, page, kv, g, lens, n, window, sinks, room):
    """Tables of the sequences' size, and with room for more (pieces)."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    _window_case(gpu, dtype, d, page, kv, g, lens, n, window, sinks, room=room)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,page,kv,g,lens,n,window,sinks", [
    (64, 16, 2, 4, [4000, 70, 1], 2, 3000, 4), (128, 64, 1, 8, [3500, 2222], 30, 1500, 100),
    (128, 16, 1, 1, [2500], 1, 2100, 0), (256, 32, 1, 4, [2600], 25, 2000, 1),
])
@pytest.mark.parametrize("rows", ROWS)
def test_long_windows(gpu, monkeypatch, rows, dtype, d, page, kv, g, lens, n, window, sinks):
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    _window_case(gpu, dtype, d, page, kv, g, lens, n, window, sinks, room=5000)


def _parents(gen, B, n, shape):
    at = torch.arange(n).expand(B, n)
    if shape == "chain":
        return at - 1
    if shape == "star":
        return torch.where(at > 0, 0, -1)
    if shape == "none":
        return torch.full((B, n), -1)
    p = (torch.rand((B, n), generator=gen) * (at + 1)).long() - 1
    if shape == "wrong":  # numbers that are no parent's
        bad = torch.tensor([-2**31, -7, 2**31 - 1, n, 300])
        p = torch.where(torch.rand((B, n), generator=gen) < 0.4,
                        bad[torch.randint(0, 5, (B, n), generator=gen)], p)
        p[:, n // 2] = n // 2                       # its own
    return p


def _tree_case(gpu, dtype, d, page, kv, g, lens, n, P, shape, scale=None, **kw):
    cache, Q, table, lens_d, prefix, gen = _setup(gpu, dtype, d, page, kv, g, lens, n, P, **kw)
    scale = 1 / math.sqrt(d) if scale is None else scale
    parents = _parents(gen, len(lens), n, shape).to(torch.int32)
    O, lse = gpu.cache_attend_tree(cache, Q.to(DEV), table.to(DEV), lens_d, parents.to(DEV),
                                   prefix=prefix, prefix_len=P, scale=scale)
    torch.cuda.synchronize()
    known = parents.tolist()
    _compare(cache, Q, table, lens, lambda b, m: tree_seen(lens[b], known[b], m), scale, O, lse,
             prefix, P)


TREES = [
    # d, page, key heads, query heads of each, lengths, drafted tokens, prefix
    (64, 16, 2, 1, [1, 5, 33, 16, 17, 0], 1, 0),
    (64, 16, 1, 4, [300, 8, 64, 65], 8, 0),
    (128, 64, 2, 4, [1000, 3, 517], 5, 77),          # one with padding
    (32, 16, 3, 1, [40, 41, 64], 33, 0),
    (96, 16, 1, 2, [290], 31, 16), (256, 256, 1, 3, [600, 20], 20, 300),
    (160, 128, 1, 1, [129], 60, 1), (192, 64, 1, 2, [64], 32, 0), (224, 16, 1, 1, [15], 9, 15),
    # many rows
    (64, 16, 1, 2, [70, 200, 33], 33, 0),
    (64, 16, 2, 1, [300, 256], 256, 0),
    (128, 64, 1, 4, [700, 100, 40], 63, 130),
    (128, 16, 1, 8, [400, 0, 11], 12, 0), (32, 16, 1, 3, [333], 100, 40),
    (96, 32, 1, 1, [140], 129, 0), (256, 128, 1, 4, [400], 40, 33), (160, 16, 1, 2, [250], 65, 0),
    (192, 16, 1, 3, [250], 31, 64), (224, 64, 1, 2, [280], 50, 0),
    (64, 16, 1, 70, [90, 17], 1, 0),
]


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("shape", ["random", "wrong"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,page,kv,g,lens,n,P", TREES)
def test_tree(gpu, monkeypatch, rows, dtype, d, page, kv, g, lens, n, P, shape):
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    _tree_case(gpu, dtype, d, page, kv, g, lens, n, P, shape)
    _tree_case(gpu, dtype, d, page, kv, g, lens, n, P, shape, room=2000, seed=1)


@pytest.mark.parametrize("shape", ["chain", "star", "none"])
@pytest.mark.parametrize("g,n", [(1, 40), (4, 40), (2, 256)])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_tree_shapes(gpu, monkeypatch, rows, shape, g, n):
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    _tree_case(gpu, torch.float16, 64, 16, 1, g, [300, 45, n], n, 0, shape)


@pytest.mark.parametrize("own", ROWS)
@pytest.mark.parametrize("rows", ["16", "128"])
@pytest.mark.parametrize("g,n", [(2, 4), (4, 30)])
def test_tree_behind_a_prefix(gpu, monkeypatch, rows, own, g, n):
    """The prefix by the kernel of 16 query rows and by that of 128, beside the own keys where
    these go by many rows."""
    monkeypatch.setenv("F3S_PREFIX_ROWS", rows)
    monkeypatch.setenv("F3S_OWN_ROWS", own)
    _tree_case(gpu, torch.bfloat16, 128, 32, 2, g, [(7 * b) % 50 for b in range(20)], n, 321,
               "random")


@pytest.mark.parametrize("rows", ["16", "128"])
def test_a_chain_is_cache_attend(gpu, monkeypatch, rows):
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    for n, g in ((5, 2), (40, 4)):
        cache, Q, table, lens, _, _ = _setup(gpu, torch.float16, 64, 16, 2, g, [200, 77], n)
        chain = (torch.arange(n, dtype=torch.int32, device=DEV) - 1).expand(2, n).contiguous()
        args = (cache, Q.to(DEV), table.to(DEV), lens)
        O, lse = gpu.cache_attend(*args)
        O2, lse2 = gpu.cache_attend_tree(*args, chain)
        O3, lse3 = gpu.cache_attend_window(*args, 10**6)
        for x, y in ((O2, lse2), (O3, lse3)):
            # (two roundings of a result, and of its probabilities)
            assert torch.allclose(O.float(), x.float(), rtol=2.0 ** -9, atol=2.0 ** -10)
            assert torch.allclose(lse, y, atol=1e-5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("spread", [6, 60])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_values_of_different_sizes(gpu, monkeypatch, rows, dtype, spread):
    """Values that differ by 2^120 (bf16): what a row sees counts, not what others do."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    spread = min(spread, 6) if dtype == torch.float16 else spread
    for n, g in ((3, 2), (40, 3)):
        _window_case(gpu, dtype, 64, 16, 1, g, [300, 90], n, 50, 3, spread=spread)
        _tree_case(gpu, dtype, 64, 16, 1, g, [300, 90], n, 33, "random", spread=spread)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 5.0])
@pytest.mark.parametrize("n,g", [(3, 2), (40, 3)])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_scales(gpu, monkeypatch, rows, scale, n, g):
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    _window_case(gpu, torch.float16, 64, 16, 1, g, [200], n, 50, 3, scale=scale)
    _tree_case(gpu, torch.float16, 64, 16, 1, g, [200], n, 33, "random", scale=scale)


@pytest.mark.parametrize("n,g", [(6, 2), (40, 3)])
@pytest.mark.parametrize("large", [2.0 ** 60, 3.0])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_what_a_token_does_not_see_changes_no_bit(gpu, monkeypatch, rows, n, g, large):
    """Other tokens' keys, values and queries, much larger or alike."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    dtype = torch.bfloat16
    lens, window, sinks = [300], 60, 2
    cache, Q, table, lens_d, _, gen = _setup(gpu, dtype, 64, 16, 1, g, lens, n)
    parents = _parents(gen, 1, n, "random").to(torch.int32)
    t = n // 2
    K, V = gpu.cache_read(cache, table.to(DEV), lens_d, 300, dtype)
    known = parents.tolist()
    for kind in ("window", "tree"):
        if kind == "window":
            seen = window_seen(300, n, 300, window, sinks)[t]
            run = lambda q: gpu.cache_attend_window(cache, q.to(DEV), table.to(DEV), lens_d,
                                                    window, sinks)
        else:
            seen = tree_seen(300, known[0], 300)[t]
            run = lambda q: gpu.cache_attend_tree(cache, q.to(DEV), table.to(DEV), lens_d,
                                                  parents.to(DEV))
        gpu.cache_write(cache, K, V, table.to(DEV), lens_d)
        O, lse = run(Q)
        K2, V2 = K.clone(), V.clone()
        for x in (K2, V2):
            x[0, ~seen.to(DEV)] *= -large
        gpu.cache_write(cache, K2, V2, table.to(DEV), lens_d)
        Q2 = -Q * 2
        Q2[0, t] = Q[0, t]
        O2, lse2 = run(Q2)
        assert torch.equal(O[0, t], O2[0, t]) and torch.equal(lse[0, t], lse2[0, t]), kind
        assert not torch.equal(O, O2)


@pytest.mark.parametrize("n,g", [(5, 2), (40, 3)])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_bad_pages_and_lengths(gpu, monkeypatch, rows, n, g):
    """Pages that are none, lengths below zero and beyond the table."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    lens = [100, 61, -5, 200, 64]
    cache, Q, table, _, _, gen = _setup(gpu, torch.float16, 64, 16, 1, g, [100, 61, 1, 112, 64],
                                        n)
    table = table.clone()
    assert table.shape[1] == 7
    table[0, 2], table[0, 6], table[1, 0], table[4] = -1, cache.n_pages, 2**31 - 1, -9
    scale = 1 / 8
    args = (cache, Q.to(DEV), table.to(DEV), _ints(lens))
    O, lse = gpu.cache_attend_window(*args, 50, 3)
    _compare(cache, Q, table, lens, lambda b, m: window_seen(lens[b], n, m, 50, 3), scale, O, lse)
    parents = _parents(gen, 5, n, "random").to(torch.int32)
    O, lse = gpu.cache_attend_tree(*args, parents.to(DEV))
    known = parents.tolist()
    _compare(cache, Q, table, lens, lambda b, m: tree_seen(lens[b], known[b], m), scale, O, lse)


@pytest.mark.parametrize("n,g", [(2, 2), (40, 2)])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_captured_with_changing_lengths(gpu, monkeypatch, rows, n, g):
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    # (every row below a length has to be there: all of 500 are written first)
    cache, Q, table, lens, _, gen = _setup(gpu, torch.float16, 64, 16, 2, g, [500, 500, 500], n,
                                           room=1500)
    q, t = Q.to(DEV), table.to(DEV)
    parents = torch.full((3, n), -1, dtype=torch.int32, device=DEV)

    def step():
        return (gpu.cache_attend_window(cache, q, t, lens, 90, 4)
                + gpu.cache_attend_tree(cache, q, t, lens, parents))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for new in ([500, 300, 64], [41, 7, 450], [0, 1, 2], [500, 500, 500]):
        lens.copy_(torch.tensor(new))
        parents.copy_(_parents(gen, 3, n, "random"))
        eager = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rows", ["16", "128"])
def test_calls_side_by_side(gpu, monkeypatch, rows):
    """On streams of their own, each with its own workspace."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    cases = [_setup(gpu, torch.float16, 64, 16, 2, 4, [1500, 900], n, seed=n) for n in (1, 30)]
    parents = [(torch.arange(n, dtype=torch.int32, device=DEV) // 2 - 1).expand(2, n).contiguous()
               for n in (1, 30)]
    calls = []
    for (cache, Q, table, lens, _, _), p in zip(cases, parents):
        q, t = Q.to(DEV), table.to(DEV)
        calls.append(lambda c=cache, q=q, t=t, m=lens, **k: gpu.cache_attend_window(
            c, q, t, m, 1000, 4, **k))
        calls.append(lambda c=cache, q=q, t=t, m=lens, p=p, **k: gpu.cache_attend_tree(
            c, q, t, m, p, **k))
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        got = [c(stream=s) for c, s in zip(calls, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_nothing_to_do_and_refusals(gpu):
    cache, Q, table, lens, _, _ = _setup(gpu, torch.float16, 64, 16, 2, 2, [50, 60], 3)
    q, t = Q.to(DEV), table.to(DEV)
    p = torch.full((2, 3), -1, dtype=torch.int32, device=DEV)
    none = torch.empty((2, 0, 4, 64), dtype=torch.float16, device=DEV)
    assert gpu.cache_attend_window(cache, none, t, lens, 5)[0].shape == none.shape
    assert gpu.cache_attend_tree(cache, none, t, lens, p[:, :0].contiguous())[1].shape == (2, 0, 4)
    for window, sinks in ((-1, 0), (5, -1), (2**31, 0)):
        with pytest.raises(ValueError):
            gpu.cache_attend_window(cache, q, t, lens, window, sinks)
    with pytest.raises(ValueError):
        gpu.cache_attend_tree(cache, q, t, lens, p[:, :2].contiguous())
    with pytest.raises(TypeError):
        gpu.cache_attend_tree(cache, q, t, lens, p.long())
    with pytest.raises(ValueError):
        gpu.cache_attend_tree(cache, q, t, lens, p, prefix_len=4)
    many = torch.zeros((2, 257, 4, 64), dtype=torch.float16, device=DEV)
    with pytest.raises(gpu.F3SError):
        gpu.cache_attend_tree(cache, many, t, lens,
                              torch.zeros((2, 257), dtype=torch.int32, device=DEV))
    with pytest.raises(gpu.F3SError):
        gpu.cache_attend_window(cache, q, t, lens, 5, out=q)
    with pytest.raises(ValueError):
        gpu.cache_attend_window(cache, q[:1], t, lens, 5)


@pytest.mark.parametrize("rows", ["16", "128"])
def test_two_steps_of_a_draft(gpu, monkeypatch, rows):
    """The operators as a step of generation uses them: pages for a tree, its rows, its
    attention, the accepted branch kept; then the next token over a window."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    B, n, page, kv, g, d, M = 3, 7, 16, 1, 2, 64, 8
    gen = torch.Generator().manual_seed(9)
    pool = gpu.PagePool.full(B * M, page, device=DEV)
    cache = _cache(gpu, B * M, page, kv, d)
    table = torch.full((B, M), -1, dtype=torch.int32, device=DEV)
    lens = _ints([0] * B)
    text = 40
    states = lambda k: [_rows(gen, (B, k, kv, d), torch.float16).to(DEV) for _ in "KV"]
    lens, slots = gpu.pages_assign(pool, table, lens, _ints([text, text - 9, text - 1]), n=1)
    assert (slots >= 0).all()
    gpu.cache_write(cache, *states(text), table, lens)
    parents = _ints([[-1, 0, 0, 1, 1, 2, 5]] * B)
    branch = _ints([[0, 2, 5, 6], [0, 1, 4, -1], [-1, -1, -1, -1]])
    for _ in range(2):
        got, _ = gpu.pages_assign(pool, table, lens, lens + n)
        gpu.cache_write(cache, *states(n), table, got)
        Q = torch.randn((B, n, kv * g, d), generator=gen, dtype=torch.float64).half()
        O, lse = gpu.cache_attend_tree(cache, Q.to(DEV), table, got, parents)
        known = parents.tolist()
        now = got.tolist()
        _compare(cache, Q, table.cpu(), now, lambda b, m: tree_seen(now[b], known[b], m), 1 / 8,
                 O, lse)
        # the last token of the branch sees the same keys after they have moved
        kept = gpu.cache_keep(cache, table, got, n, branch)
        lens, _ = gpu.pages_assign(pool, table, got, kept)
        for b, last in ((0, 6), (1, 4)):
            q = Q[b: b + 1, last: last + 1].to(DEV)
            O2, lse2 = gpu.cache_attend(cache, q, table[b: b + 1], lens[b: b + 1])
            assert torch.allclose(O2[0, 0].float(), O[b, last].float(), atol=2.0 ** -9)
            assert torch.allclose(lse2[0, 0], lse[b, last], atol=1e-5)
        now = lens.tolist()
        Q = torch.randn((B, 1, kv * g, d), generator=gen, dtype=torch.float64).half()
        O, lse = gpu.cache_attend_window(cache, Q.to(DEV), table, lens, 16, 2)
        _compare(cache, Q, table.cpu(), now, lambda b, m: window_seen(now[b], 1, m, 16, 2), 1 / 8,
                 O, lse)
    assert lens.tolist() == [text + 8, text - 9 + 6, text - 1]
