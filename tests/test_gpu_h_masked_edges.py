"""Edges of the window, the trees, the moving of accepted tokens and the page tables:
offsets beyond 32 bits, tensors at odd places, results that are given, what lies behind the
last row."""
import math

import pytest
import torch

from _dense import attention, close, half_step
from test_gpu_e_window import seen_keys
from test_gpu_g_masked import tree_seen, window_seen

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_window_of_keys_beyond_4_gib(gpu):
    """The newest tokens of a sequence whose keys take 4.5 GB: its window and its sinks."""
    n, nq, kv, d, W, S = 2_200_000, 37, 8, 128, 500, 3
    gen = torch.Generator(device=DEV).manual_seed(1)
    K, V = (torch.empty((n, kv, d), dtype=torch.float16, device=DEV) for _ in "KV")
    for x in (K, V):
        x.normal_(generator=gen)
    Q, G = (torch.randn((nq, 2 * kv, d), generator=gen, device=DEV).half() for _ in "QG")
    plan = gpu.WindowPlan([0, nq], [0, n], 2 * kv, kv, d, window=W, sinks=S, device=DEV)
    O, lse = gpu.window_forward(plan, Q, K, V)
    dQ, dK, dV = gpu.window_backward(plan, Q, K, V, O, G, lse)
    first = n - nq - W
    at = torch.cat([torch.arange(S), torch.arange(first, n)])
    seen = torch.cat([torch.ones((nq, S), dtype=torch.bool), seen_keys(nq, nq + W, W, 0)], 1)
    u = half_step(torch.float16)
    for h in (0, 5, 15):
        f = attention(Q[:, h].double().cpu(), K[at.to(DEV), h // 2].double().cpu(),
                      V[at.to(DEV), h // 2].double().cpu(), 1 / math.sqrt(d), u, seen=seen)
        close(O[:, h], f["O"], f["O_tol"], h)
        close(lse[:, h], f["lse"], f["lse_tol"], h)
    # gradients lie where keys are seen, and nowhere else
    keys = torch.zeros(n, dtype=torch.bool, device=DEV)
    keys[at.to(DEV)] = seen.any(0).to(DEV)
    for x in (dK, dV):
        there = x.view(n, -1).ne(0).any(1)
        assert torch.equal(there, keys)
    # dV's sums: every query's probabilities add up to 1
    want = G.double().view(nq, kv, 2, d).sum((0, 2)).cpu()
    got = dV[at.to(DEV)].double().sum(0).cpu()
    spread = G.double().abs().view(nq, kv, 2, d).sum((0, 2)).cpu()
    # (the probabilities' and the results' roundings, 2^-11 each, and twice that of lse)
    assert bool(((got - want).abs() <= 4 * u * spread).all())


@pytest.mark.parametrize("rows", ["16", "128"])
def test_cache_rows_beyond_4_gib(gpu, monkeypatch, rows):
    """Pages whose codes lie beyond 4 GiB: written, attended to, moved."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    kv, page, d = 8, 64, 128
    n_pages = 80_000                    # 5.2 GB of codes
    cache = gpu.Cache.empty(n_pages, page, kv, d, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(2)
    n, g = 40, 2
    table = _ints([[n_pages - 1, 3, n_pages - 2, 70_001], [5, n_pages - 7, 6, 66_000]])
    lens = _ints([250, 200])
    K, V = (torch.randn((2, 250, kv, d), generator=gen, device=DEV).half() for _ in "KV")
    gpu.cache_write(cache, K, V, table, lens)
    K, V = gpu.cache_read(cache, table, lens, 250, torch.float32)
    parents = torch.arange(n, dtype=torch.int32, device=DEV).sub(2).clamp(min=-1).expand(
        2, n).contiguous()
    known = parents.tolist()
    for m in (1, n):                    # by 16 rows and by 128
        Q = torch.randn((2, m, kv * g, d), generator=gen, device=DEV).half()
        got = {"window": gpu.cache_attend_window(cache, Q, table, lens, 90, 3),
               "tree": gpu.cache_attend_tree(cache, Q, table, lens, parents[:, :m].contiguous())}
        for b, length in enumerate(lens.tolist()):
            k, v = (x[b, 250 - length:].double().cpu() for x in (K, V))
            for what, (O, lse) in got.items():
                seen = window_seen(length, m, length, 90, 3) if what == "window" else \
                    tree_seen(length, known[b][:m], length)
                for h in (0, 9, 15):
                    f = attention(Q[b, :, h].double().cpu(), k[:, h // g], v[:, h // g],
                                  1 / math.sqrt(d), half_step(torch.float16), seen=seen)
                    tol = f["O_tol"] + 2.0 ** -24 * float(v.abs().max()) * length
                    close(O[b, :, h], f["O"], tol, (what, m, b, h))
                    close(lse[b, :, h], f["lse"], f["lse_tol"], (what, m, b, h))
    picks = _ints([[1, 7, 8, 30], [0, 2, 39, -1]])
    new = gpu.cache_keep(cache, table, lens, n, picks)
    assert new.tolist() == [214, 163]
    K2, V2 = gpu.cache_read(cache, table, new, 214, torch.float32)
    for a, b in ((K, K2), (V, V2)):
        assert torch.equal(b[0, :210], a[0, :210]) and torch.equal(b[1, 51:211], a[1, 50:210])
        assert torch.equal(b[0, 210:], a[0, 210 + torch.tensor([1, 7, 8, 30], device=DEV)])
        assert torch.equal(b[1, 211:], a[1, 210 + torch.tensor([0, 2, 39], device=DEV)])


def test_a_pool_with_slots_beyond_32_bits(gpu):
    page, n_pages = 256, 9_000_000       # 2.3e9 places
    pool = gpu.PagePool.full(n_pages, page, device=DEV)
    table = torch.full((1, 8), -1, dtype=torch.int32, device=DEV)
    got, slots = gpu.pages_assign(pool, table, _ints([0]), _ints([2000]), n=3)
    assert got.tolist() == [2000] and int(pool.count) == n_pages - 8
    assert slots.tolist() == [[(n_pages - 1) * page + 1997 - 7 * page + t for t in range(3)]]


@pytest.mark.parametrize("d,kv,g", [(64, 2, 2), (128, 1, 4), (96, 1, 1)])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_given_results_and_what_lies_beside_them(gpu, monkeypatch, rows, d, kv, g):
    """Results into rows of larger buffers: what stands before and behind stays."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    n, H = 150, kv * g
    gen = torch.Generator(device=DEV).manual_seed(3)
    Q = torch.randn((n, H, d), generator=gen, device=DEV).half()
    K, V = (torch.randn((n, kv, d), generator=gen, device=DEV).half() for _ in "KV")
    plan = gpu.WindowPlan([0, 70, n], [0, 70, n], H, kv, d, window=33, sinks=2, device=DEV)
    want = gpu.window_forward(plan, Q, K, V)
    big = torch.full((n + 20, H, d), 7.0, dtype=torch.float16, device=DEV)
    stats = torch.full((n + 20, H), 7.0, device=DEV)
    out, lse = gpu.window_forward(plan, Q, K, V, out=big[10:-10], lse=stats[10:-10])
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert bool((big[:10] == 7).all() and (big[-10:] == 7).all())
    assert bool((stats[:10] == 7).all() and (stats[-10:] == 7).all())
    cache = gpu.Cache.empty(40, 16, kv, d, device=DEV)
    table = torch.arange(40, dtype=torch.int32, device=DEV).view(2, 20)
    lens = _ints([200, 111])
    x = [torch.randn((2, 200, kv, d), generator=gen, device=DEV).half() for _ in "KV"]
    gpu.cache_write(cache, *x, table, lens)
    for m in (3, 70):
        Q = torch.randn((2, m, H, d), generator=gen, device=DEV).half()
        p = torch.zeros((2, m), dtype=torch.int32, device=DEV)
        for call in (lambda **k: gpu.cache_attend_window(cache, Q, table, lens, 40, 1, **k),
                     lambda **k: gpu.cache_attend_tree(cache, Q, table, lens, p, **k)):
            want = call()
            big = torch.full((4, m, H, d), 7.0, dtype=torch.float16, device=DEV)
            stats = torch.full((4, m, H), 7.0, device=DEV)
            out, lse = call(out=big[1:3], lse=stats[1:3])
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            assert bool((big[0] == 7).all() and (big[3] == 7).all())
            assert bool((stats[0] == 7).all() and (stats[3] == 7).all())


def test_pages_beside_others_stay(gpu):
    """Rows of a table and a pool that are parts of larger tensors."""
    room = torch.full((12, 6), 77, dtype=torch.int32, device=DEV)
    list_ = torch.full((40,), 99, dtype=torch.int32, device=DEV)
    list_[8:32] = torch.arange(24)
    pool = gpu.PagePool(list_[8:32], _ints([24]), 16)
    lens, table = _ints([0, 0, 0]), room[4:7]
    got, _ = gpu.pages_assign(pool, table, lens, _ints([40, 96, 1]))
    back, _ = gpu.pages_assign(pool, table, got, lens)
    assert back.tolist() == [0, 0, 0] and int(pool.count) == 24
    assert bool((room[:4] == 77).all() and (room[7:] == 77).all())
    assert bool((list_[:8] == 99).all() and (list_[32:] == 99).all())
    assert list_[8:32].tolist() == list(range(24))
    assert room[4].tolist()[3:] == [77] * 3       # entries that no length reached


def test_large_scores(gpu):
    """Scores that 32 bits hold in steps: the largest probability is 1 all the same."""
    n, d = 200, 64
    gen = torch.Generator(device=DEV).manual_seed(4)
    Q, K = (torch.randn((n, 1, d), generator=gen, device=DEV).mul(30000).to(torch.bfloat16)
            for _ in "QK")
    V = torch.randn((n, 1, d), generator=gen, device=DEV).to(torch.bfloat16)
    plan = gpu.WindowPlan([0, n], [0, n], 1, 1, d, window=40, sinks=2, device=DEV)
    O, _ = gpu.window_forward(plan, Q, K, V, scale=100.0)
    x = (Q[:, 0].double() @ K[:, 0].double().T).cpu()
    x = torch.where(seen_keys(n, n, 40, 2), x, -math.inf)
    top = x.argmax(1)
    # (a runner-up within 2^-20 of the largest score would share the probability)
    second = x.clone().scatter_(1, top[:, None], -math.inf).amax(1)
    alone = second < x.amax(1) - 2.0 ** -18 * x.abs().nan_to_num(0, posinf=0, neginf=0).amax(1)
    assert int(alone.sum()) > 150
    assert torch.equal(O[alone.to(DEV), 0], V[top[alone].to(DEV), 0])


@pytest.mark.parametrize("what", ["window", "tree"])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_thousands_of_sequences(gpu, monkeypatch, rows, what):
    """More than the kernels divide one by one."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    B, kv, d, page = 9000, 1, 32, 16
    gen = torch.Generator(device=DEV).manual_seed(5)
    cache = gpu.Cache.empty(B * 7, page, kv, d, device=DEV)
    table = torch.randperm(B * 7, generator=gen, device=DEV).to(torch.int32).view(B, 7)
    lens = torch.randint(0, 113, (B,), generator=gen, device=DEV, dtype=torch.int32)
    x = [torch.randn((B, 112, kv, d), generator=gen, device=DEV).half() for _ in "KV"]
    gpu.cache_write(cache, *x, table, lens)
    Q = torch.randn((B, 2, 2, d), generator=gen, device=DEV).half()
    chain = _ints([[-1, 0]]).expand(B, 2).contiguous()
    if what == "window":
        O, lse = gpu.cache_attend_window(cache, Q, table, lens, 1000)
    else:
        O, lse = gpu.cache_attend_tree(cache, Q, table, lens, chain)
    want, ref = gpu.cache_attend(cache, Q, table, lens)
    assert torch.allclose(O.float(), want.float(), rtol=2.0 ** -9, atol=2.0 ** -10)
    assert torch.allclose(lse, ref, atol=1e-5) or bool(
        ((lse - ref).abs() < 1e-5).logical_or(lse == ref).all())


def test_many_rows_of_thousands_of_sequences(gpu):
    """A tree's kernel of many rows where every sequence is one item."""
    B, kv, d, page, n = 8300, 1, 32, 16, 65
    gen = torch.Generator(device=DEV).manual_seed(6)
    cache = gpu.Cache.empty(600, page, kv, d, device=DEV)
    table = torch.randint(0, 600, (B, 20), generator=gen, device=DEV, dtype=torch.int32)
    lens = torch.randint(65, 321, (B,), generator=gen, device=DEV, dtype=torch.int32)
    K, V = (torch.randn((1, 9600, kv, d), generator=gen, device=DEV).half() for _ in "KV")
    gpu.cache_write(cache, K, V, torch.arange(600, dtype=torch.int32, device=DEV).view(1, -1),
                    _ints([9600]))
    Q = torch.randn((B, n, 1, d), generator=gen, device=DEV).half()
    chain = (torch.arange(n, dtype=torch.int32, device=DEV) - 1).expand(B, n).contiguous()
    O, lse = gpu.cache_attend_tree(cache, Q, table, lens, chain)
    want, ref = gpu.cache_attend(cache, Q, table, lens)
    assert torch.allclose(O.float(), want.float(), rtol=2.0 ** -9, atol=2.0 ** -10)
    assert torch.allclose(lse, ref, atol=1e-5)


@pytest.mark.parametrize("rows", ["16", "128"])
def test_two_graphs_of_one_cache(gpu, monkeypatch, rows):
    """Captured apart, replayed in any order: neither shares memory with the other."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    B, n, kv, d = 3, 20, 1, 64
    gen = torch.Generator(device=DEV).manual_seed(7)
    cache = gpu.Cache.empty(300, 16, kv, d, device=DEV)
    table = torch.arange(300, dtype=torch.int32, device=DEV).view(B, 100)
    lens = _ints([1600, 900, 33])
    x = [torch.randn((B, 1600, kv, d), generator=gen, device=DEV).half() for _ in "KV"]
    gpu.cache_write(cache, *x, table, lens)
    Q = torch.randn((B, n, 4, d), generator=gen, device=DEV).half()
    p = (torch.arange(n, dtype=torch.int32, device=DEV) // 3 - 1).expand(B, n).contiguous()
    calls = [lambda: gpu.cache_attend_window(cache, Q, table, lens, 1200, 4),
             lambda: gpu.cache_attend_tree(cache, Q, table, lens, p)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(c())
        graphs.append(graph)
    for order in ((0, 1), (1, 0), (1, 1, 0)):
        for o in outs:
            o[0].zero_()
            o[1].zero_()
        for k in order:
            graphs[k].replay()
        calls[0]()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
