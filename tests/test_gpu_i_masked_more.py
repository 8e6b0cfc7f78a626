"""More of attention over the 8-bit cache with a window or a tree of drafted tokens, on the GPU
against plain 64-bit attention: trees that end inside a tile of keys, prefixes by many rows at
every head size, the kernel of 256 rows at the edges."""
import math

import pytest
import torch

from test_gpu_g_masked import (_compare, _ints, _parents, _setup, _tree_case, _window_case,
                               tree_seen, window_seen)

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
WIDE = [96, 128]  # head sizes that have the kernel of 256 rows


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [225, 256])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_trees_that_end_inside_a_tile(gpu, monkeypatch, rows, n, d):
    """The last tile's second half lies behind the last token that a tree can have."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    _tree_case(gpu, torch.float16, d, 16, 1, 1, [257, 288, 321, 10, 230], n, 0, "random")
    _tree_case(gpu, torch.float16, d, 16, 1, 1, [257, 288, 321, 10, 230], n, 33, "random")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("P", [1, 20, 32, 33, 321])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_prefixes_beside_the_own_keys(gpu, monkeypatch, d, P, dtype):
    """A prefix in the launch of the own keys: of one tile, of a few, of pieces."""
    monkeypatch.setenv("F3S_PREFIX_ROWS", "128")
    for rows in ["128", "256"] if d in WIDE else ["128"]:
        monkeypatch.setenv("F3S_OWN_ROWS", rows)
        _tree_case(gpu, dtype, d, 16, 2, 3, [60, 0, 131, 9], 25, P, "random")
        _tree_case(gpu, dtype, d, 64, 1, 3, [70], 61, P, "random", room=1500)


@pytest.mark.parametrize("d", WIDE)
def test_many_rows_by_the_rule(gpu, monkeypatch, d):
    """4,096 rows of a key head and more, none forced."""
    monkeypatch.delenv("F3S_OWN_ROWS", raising=False)
    monkeypatch.delenv("F3S_PREFIX_ROWS", raising=False)
    _window_case(gpu, torch.bfloat16, d, 64, 1, 4, [1300], 1030, 400, 5)
    _tree_case(gpu, torch.float16, d, 16, 1, 16, [400], 256, 0, "random")
    _tree_case(gpu, torch.float16, d, 16, 1, 16, [257], 256, 1700, "random")


def _both(gpu, dtype, d, g, lens, n, window, sinks, P, **kw):
    _window_case(gpu, dtype, d, 16, 1, g, lens, n, window, sinks, **kw)
    _tree_case(gpu, dtype, d, 16, 1, g, lens, n, P, "random", **kw)


@pytest.mark.parametrize("d", WIDE)
@pytest.mark.parametrize("spread", [6, 60])
def test_values_of_different_sizes(gpu, monkeypatch, d, spread):
    monkeypatch.setenv("F3S_OWN_ROWS", "256")
    dtype = torch.float16 if spread == 6 else torch.bfloat16
    _both(gpu, dtype, d, 3, [300, 90], 100, 50, 3, 33, spread=spread)


@pytest.mark.parametrize("d", WIDE)
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 5.0])
def test_scales(gpu, monkeypatch, d, scale):
    monkeypatch.setenv("F3S_OWN_ROWS", "256")
    _both(gpu, torch.float16, d, 3, [200], 100, 50, 3, 33, scale=scale)


@pytest.mark.parametrize("d", WIDE)
def test_bad_pages_and_lengths(gpu, monkeypatch, d):
    """Pages that are none, lengths below zero and beyond the table."""
    monkeypatch.setenv("F3S_OWN_ROWS", "256")
    lens, n = [100, 61, -5, 200, 64], 100
    cache, Q, table, _, _, gen = _setup(gpu, torch.float16, d, 16, 1, 3, [100, 61, 1, 112, 64], n)
    table = table.clone()
    table[0, 2], table[0, 6], table[1, 0], table[4] = -1, cache.n_pages, 2**31 - 1, -9
    scale = 1 / math.sqrt(d)
    args = (cache, Q.to(DEV), table.to(DEV), _ints(lens))
    O, lse = gpu.cache_attend_window(*args, 50, 3)
    _compare(cache, Q, table, lens, lambda b, m: window_seen(lens[b], n, m, 50, 3), scale, O, lse)
    parents = _parents(gen, 5, n, "random").to(torch.int32)
    O, lse = gpu.cache_attend_tree(*args, parents.to(DEV))
    known = parents.tolist()
    _compare(cache, Q, table, lens, lambda b, m: tree_seen(lens[b], known[b], m), scale, O, lse)


@pytest.mark.parametrize("d", WIDE)
@pytest.mark.parametrize("large", [2.0 ** 60, 3.0])
def test_what_a_token_does_not_see_changes_no_bit(gpu, monkeypatch, d, large):
    monkeypatch.setenv("F3S_OWN_ROWS", "256")
    dtype, n, g, m = torch.bfloat16, 100, 3, 300
    cache, Q, table, lens, _, gen = _setup(gpu, dtype, d, 16, 1, g, [m], n)
    parents = _parents(gen, 1, n, "random").to(torch.int32)
    K, V = gpu.cache_read(cache, table.to(DEV), lens, m, dtype)
    for t in (0, n // 2, n - 1):
        for seen, run in (
                (window_seen(m, n, m, 60, 2)[t],
                 lambda q: gpu.cache_attend_window(cache, q.to(DEV), table.to(DEV), lens, 60, 2)),
                (tree_seen(m, parents.tolist()[0], m)[t],
                 lambda q: gpu.cache_attend_tree(cache, q.to(DEV), table.to(DEV), lens,
                                                 parents.to(DEV)))):
            gpu.cache_write(cache, K, V, table.to(DEV), lens)
            O, lse = run(Q)
            K2, V2 = K.clone(), V.clone()
            for x in (K2, V2):
                x[0, ~seen.to(DEV)] *= -large
            gpu.cache_write(cache, K2, V2, table.to(DEV), lens)
            Q2 = -Q * 2
            Q2[0, t] = Q[0, t]
            O2, lse2 = run(Q2)
            assert torch.equal(O[0, t], O2[0, t]) and torch.equal(lse[0, t], lse2[0, t])
            assert not torch.equal(O, O2)


@pytest.mark.parametrize("d", WIDE)
def test_captured_and_on_other_streams(gpu, monkeypatch, d):
    """A step replayed while lengths and trees change, and beside others on their own streams."""
    monkeypatch.setenv("F3S_OWN_ROWS", "256")
    monkeypatch.setenv("F3S_PREFIX_ROWS", "128")
    n, P = 100, 77
    cache, Q, table, lens, prefix, gen = _setup(gpu, torch.float16, d, 16, 2, 3, [500] * 3, n, P,
                                                room=1500)
    q, t = Q.to(DEV), table.to(DEV)
    parents = _parents(gen, 3, n, "random").to(torch.int32).to(DEV)

    def window(**kw):
        return gpu.cache_attend_window(cache, q, t, lens, 90, 4, **kw)

    def tree(**kw):
        return gpu.cache_attend_tree(cache, q, t, lens, parents, prefix=prefix, prefix_len=P, **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        window(), tree()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = window() + tree()
    streams = [torch.cuda.Stream() for _ in range(4)]
    for new in ([500, 300, 64], [41, 7, 450], [0, 1, 2], [500, 500, 500]):
        lens.copy_(torch.tensor(new))
        parents.copy_(_parents(gen, 3, n, "random"))
        want = window() + tree()
        graph.replay()
        torch.cuda.synchronize()
        got = [call(stream=s) for call, s in zip((window, tree) * 2, streams)]
        torch.cuda.synchronize()
        for x in (out, got[0] + got[1], got[2] + got[3]):
            for a, b in zip(x, want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("B", [1024, 1025])
def test_as_many_sequences_as_are_divided_and_one_more(gpu, monkeypatch, B):
    """A chain of tokens is plain causal attention, also where one sequence is much longer."""
    monkeypatch.delenv("F3S_OWN_ROWS", raising=False)
    kv, d, page, n, room = 1, 32, 16, 33, 5000
    gen = torch.Generator(device=DEV).manual_seed(8)
    pages = -(-room // page)
    cache = gpu.Cache.empty(pages, page, kv, d, device=DEV)
    table = torch.randint(0, pages, (B, pages), generator=gen, device=DEV, dtype=torch.int32)
    lens = torch.randint(0, 300, (B,), generator=gen, device=DEV, dtype=torch.int32)
    lens[B // 2] = room
    states = [torch.randn((1, pages * page, kv, d), generator=gen, device=DEV).half()
              for _ in "KV"]
    gpu.cache_write(cache, *states, torch.arange(pages, dtype=torch.int32, device=DEV).view(1, -1),
                    _ints([pages * page]))
    Q = torch.randn((B, n, 2, d), generator=gen, device=DEV).half()
    chain = (torch.arange(n, dtype=torch.int32, device=DEV) - 1).expand(B, n).contiguous()
    O, lse = gpu.cache_attend_tree(cache, Q, table, lens, chain)
    want, ref = gpu.cache_attend(cache, Q, table, lens)
    # Of each of two kernels: a result's rounding, and its probabilities', which weigh V; of
    # lse, what 32 sums of a score in 32 bits lose (a sum of probabilities loses less).
    u = 2.0 ** -11
    K, V = gpu.cache_read(cache, table[B // 2: B // 2 + 1], lens[B // 2: B // 2 + 1], room,
                          torch.float32)
    top = max(float(x.abs().max()) for x in (V, states[1]))
    score = float(Q.float().norm(dim=3).max()) * max(
        float(x.float().norm(dim=3).max()) for x in (K, states[0])) * 2 / d ** 0.5
    assert torch.allclose(O.float(), want.float(), rtol=2 * u, atol=2 * u * top)
    assert torch.allclose(lse, ref, rtol=0, atol=2 * d * 2.0 ** -24 * score)
