"""The dense operators where they can go wrong: bad pages and lengths, powers far
apart, scales of any sign, other streams, captured graphs whose lengths change,
calls that overlap, tables beyond 4 GiB, and a decoder's steps with all of them
together."""
import math

import pytest
import torch

from _dense import attention, close, gradients, half_step, tiny
from test_gpu_b_cache import TYPES, _attend_case, _cache, _compare, _rows, _table, _values
from test_gpu_b_cross import _case, _sums

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.fixture(params=["16", "128"])
def prefix_rows(request, monkeypatch):
    monkeypatch.setenv("F3S_PREFIX_ROWS", request.param)
    return request.param


# ---- pages and lengths -----------------------------------------------------------

BAD = [-1, -2147483648, 2147483647]


@pytest.mark.parametrize("page", [16, 32, 64])
def test_bad_pages(gpu, prefix_rows, page):
    """Pages that are none: not written, zeros, and no part in attention."""
    gen = torch.Generator().manual_seed(page)
    dtype, kv, d, n = torch.bfloat16, 2, 64, 3
    lens, P = [5 * page, 3 * page + 5, 2 * page, page], 3 * page + 7
    table, n_pages = _table(gen, 4, 6, first=4)
    table[0, 1], table[0, 4], table[1, 0], table[2, :], table[3, 0] = BAD[0], BAD[1], BAD[2], -7, n_pages
    prefix = torch.tensor([1, -1, 0, 2], dtype=torch.int32)
    cache = _cache(gpu, n_pages, page, kv, d)
    top = max(lens)
    x = [_rows(gen, (4, top, kv, d), dtype) for _ in "KV"]
    gpu.cache_write(cache, x[0].to(DEV), x[1].to(DEV), table.to(DEV), _int32(lens))
    y = [_rows(gen, (1, P, kv, d), dtype) for _ in "KV"]
    gpu.cache_write(cache, y[0].to(DEV), y[1].to(DEV), prefix.view(1, -1).to(DEV), _int32([P]))
    back = gpu.cache_read(cache, table.to(DEV), _int32(lens), top, torch.float32)
    for b, m in enumerate(lens):
        for t in range(top):
            p = m - top + t
            bad = p < 0 or not 0 <= int(table[b, p // page]) < n_pages
            for got in back:
                assert bool((got[b, t] == 0).all()) == bad
    Q = torch.randn((4, n, kv * 4, d), generator=gen).to(dtype)
    O, lse = gpu.cache_attend(cache, Q.to(DEV), table.to(DEV), _int32(lens),
                              prefix=prefix.to(DEV), prefix_len=P)
    _compare(cache, Q, table, lens, prefix, P, 0.125, O, lse)
    # all of a prefix's pages bad, and all own ones: no key at all
    none = torch.full((4,), -1, dtype=torch.int32, device=DEV)
    O, lse = gpu.cache_attend(cache, Q[2:3].to(DEV), table[2:3].to(DEV), _int32([2 * page]),
                              prefix=none, prefix_len=P)
    assert not O.any() and bool((lse == -math.inf).all())


def test_lengths_that_cannot_be(gpu, prefix_rows):
    """Negative lengths count as none, and lengths beyond the table leave what is
    behind it out."""
    gen = torch.Generator().manual_seed(3)
    dtype, kv, d, page, n = torch.float16, 1, 64, 16, 4
    table, n_pages = _table(gen, 6, 3, first=2)
    cap = 3 * page
    cache = _cache(gpu, n_pages, page, kv, d, fill=0)
    x = [_rows(gen, (6, cap, kv, d), dtype).to(DEV) for _ in "KV"]
    gpu.cache_write(cache, *x, table.to(DEV), _int32([cap] * 6))
    y = [_rows(gen, (1, 20, kv, d), dtype).to(DEV) for _ in "KV"]
    prefix = torch.tensor([0, 1], dtype=torch.int32)
    gpu.cache_write(cache, *y, prefix.view(1, -1).to(DEV), _int32([20]))
    before = _values(cache)
    lens = [-1, -2147483648, cap + 1, cap + 3, 2147483647, cap]
    Q = torch.randn((6, n, 2, d), generator=gen).to(dtype)
    O, lse = gpu.cache_attend(cache, Q.to(DEV), table.to(DEV), _int32(lens),
                              prefix=prefix.to(DEV), prefix_len=20)
    _compare(cache, Q, table, lens, prefix, 20, 0.125, O, lse)
    # writing there changes nothing but what lies within
    z = [_rows(gen, (6, 2, kv, d), dtype).to(DEV) for _ in "KV"]
    gpu.cache_write(cache, *z, table.to(DEV), _int32([-1, -5, cap + 2, cap + 9, 2147483647, 0]))
    for a, b in zip(before, _values(cache)):
        assert torch.equal(a, b)
    back = gpu.cache_read(cache, table.to(DEV), _int32([-1, 0, cap + 1, 2147483647, cap, 1]), 2)
    for got in back:
        assert not got[0].any() and not got[1].any() and not got[3].any()
        assert got[2, 0].any() and not got[2, 1].any() and got[4].all()
        assert not got[5, 0].any() and got[5, 1].any()


def test_pages_that_sequences_share(gpu):
    """The same page in several tables, and twice in one, is read in each place."""
    gen = torch.Generator().manual_seed(5)
    cache = _cache(gpu, 5, 16, 2, 64)
    all_pages = torch.arange(5, dtype=torch.int32).view(1, -1)
    x = [_rows(gen, (1, 80, 2, 64), torch.bfloat16).to(DEV) for _ in "KV"]
    gpu.cache_write(cache, *x, all_pages.to(DEV), _int32([80]))
    table = torch.tensor([[3, 3, 1], [1, 3, 0], [4, 4, 4]], dtype=torch.int32)
    lens = [40, 48, 33]
    Q = torch.randn((3, 1, 4, 64), generator=gen).to(torch.bfloat16)
    O, lse = gpu.cache_attend(cache, Q.to(DEV), table.to(DEV), _int32(lens))
    _compare(cache, Q, table, lens, None, 0, 0.125, O, lse)


@pytest.mark.parametrize("dtype", TYPES)
def test_no_sequences_and_no_tokens(gpu, dtype):
    cache = _cache(gpu, 2, 16, 1, 64)
    for B, n in ((0, 1), (2, 0)):
        table, lens = torch.zeros((B, 3), dtype=torch.int32, device=DEV), _int32([4] * B)
        K = torch.zeros((B, n, 1, 64), dtype=dtype, device=DEV)
        gpu.cache_write(cache, K, K.clone(), table, lens)
        assert gpu.cache_read(cache, table, lens, n, dtype)[0].shape == (B, n, 1, 64)
        O, lse = gpu.cache_attend(cache, K.expand(B, n, 3, 64).contiguous(), table, lens)
        assert O.shape == (B, n, 3, 64) and lse.shape == (B, n, 3)
    plan = gpu.CrossPlan([0], [0], 2, 2, 64)
    E = torch.empty((0, 2, 64), dtype=dtype, device=DEV)
    O, lse = gpu.cross_forward(plan, E, E, E)
    assert all(x.shape == (0, 2, 64) for x in (O,) + gpu.cross_backward(plan, E, E, E, O, E, lse))
    # queries without keys, and keys without queries
    plan = gpu.CrossPlan([0, 3, 3], [0, 0, 5], 2, 1, 64)
    Q, K = (torch.randn(s, device=DEV).to(dtype) for s in ((3, 2, 64), (5, 1, 64)))
    O, lse = gpu.cross_forward(plan, Q, K, K)
    assert not O.any() and bool((lse == -math.inf).all())
    for x in gpu.cross_backward(plan, Q, K, K, O, Q, lse):
        assert not x.any()
    # a table without pages
    O, lse = gpu.cache_attend(cache, Q.view(3, 1, 2, 64), torch.zeros((3, 0), dtype=torch.int32,
                                                                     device=DEV), _int32([0, 4, 9]))
    assert not O.any() and bool((lse == -math.inf).all())


# ---- values ------------------------------------------------------------------------

@pytest.mark.parametrize("spread", [3.0, 12.0])
@pytest.mark.parametrize("dtype", TYPES)
def test_powers_far_apart(gpu, prefix_rows, dtype, spread):
    """Rows whose sizes differ by many powers of two, in K and in V, growing and
    shrinking along the keys."""
    gen = torch.Generator().manual_seed(int(spread))
    kv, d, page, P, m = 2, 64, 16, 200, 150
    shared, own = -(-P // page), -(-m // page)
    cache = _cache(gpu, shared + 3 * own, page, kv, d)
    prefix = torch.arange(shared, dtype=torch.int32)
    table = (shared + torch.arange(3 * own, dtype=torch.int32)).view(3, own)
    for pages, B, n in ((prefix.view(1, -1), 1, P), (table, 3, m)):
        x = [torch.randn((B, n, kv, d), generator=gen) for _ in "KV"]
        size = torch.exp2(torch.randn((2, B, n, kv, 1), generator=gen) * spread / 3)
        ramp = torch.exp2(torch.linspace(-spread, spread, n)).view(1, n, 1, 1)
        x[0] = x[0] * size[0].clamp(max=4)      # (scores of a sensible size)
        x[1] = x[1] * size[1] * ramp
        x = [v.clamp(-6e4, 6e4).to(dtype).to(DEV) for v in x]
        gpu.cache_write(cache, *x, pages.to(DEV), _int32([n] * B))
    lens = [m, m - 1, 70]
    Q = torch.randn((3, 2, kv * 4, d), generator=gen).to(dtype)
    O, lse = gpu.cache_attend(cache, Q.to(DEV), table.to(DEV), _int32(lens),
                              prefix=prefix.to(DEV), prefix_len=P)
    _compare(cache, Q, table, lens, prefix, P, 0.125, O, lse)


@pytest.mark.parametrize("scale", [0.0, -0.125, 2.0, 1e-30])
def test_scales(gpu, prefix_rows, monkeypatch, scale):
    monkeypatch.setenv("F3S_CROSS_ROWS", prefix_rows)
    _attend_case(gpu, torch.bfloat16, 64, 16, 1, 4, [33, 1, 70, 0], 2, 50, scale=scale)
    _case(gpu, torch.float16, 64, 1, 2, [40, 3], [70, 33], scale=scale)
    _case(gpu, torch.bfloat16, 96, 1, 1, [5, 60], [64, 100], scale=scale)


def test_scores_far_apart(gpu, prefix_rows, monkeypatch):
    """A few keys outweigh all others by far more than 2^6, late and early: the
    running maximum moves on, and old sums become nothing."""
    monkeypatch.setenv("F3S_CROSS_ROWS", prefix_rows)
    for scale in (8.0, 30.0):
        _attend_case(gpu, torch.float16, 64, 16, 1, 2, [300, 257], 1, 400, scale=scale, seed=9)
        _case(gpu, torch.bfloat16, 64, 2, 1, [33, 5], [400, 129], scale=scale, grad=False, seed=9)


def test_differences(gpu):
    """Gradients against differences of the 64-bit forward along directions."""
    torch.manual_seed(1)
    q_len, k_len, H, kv, d = [5, 40], [33, 70], 4, 2, 64
    q_ptr, k_ptr = _sums(q_len), _sums(k_len)
    dtype, u = torch.float16, half_step(torch.float16)
    Q, G = (torch.randn((q_ptr[-1], H, d)).to(dtype) for _ in "QG")
    K, V = (torch.randn((k_ptr[-1], kv, d)).to(dtype) for _ in "KV")
    plan = gpu.CrossPlan(q_ptr, k_ptr, H, kv, d, device=DEV)
    dev = [x.to(DEV) for x in (Q, K, V, G)]
    O, lse = gpu.cross_forward(plan, *dev[:3])
    got = [x.double().cpu() for x in gpu.cross_backward(plan, *dev[:3], O, dev[3], lse)]

    def loss(q, k, v):
        out = 0.0
        for b in range(2):
            i, j = slice(q_ptr[b], q_ptr[b + 1]), slice(k_ptr[b], k_ptr[b + 1])
            for h in range(H):
                p = torch.softmax(q[i, h] @ k[j, h // 2].T / 8, 1)
                out += float((p @ v[j, h // 2] * G[i, h].double()).sum())
        return out

    tol = [torch.zeros(x.shape, dtype=torch.float64) for x in (Q, K, K)]
    for b in range(2):
        i, j = slice(q_ptr[b], q_ptr[b + 1]), slice(k_ptr[b], k_ptr[b + 1])
        for h in range(H):
            a = [x.double() for x in (Q[i, h], K[j, h // 2], V[j, h // 2], G[i, h])]
            f = attention(*a[:3], 0.125, u)
            r = gradients(*a, 0.125, u, f)
            tol[0][i, h] = r["dQ_tol"]
            tol[1][j, h // 2] += r["dK_tol"]
            tol[2][j, h // 2] += r["dV_tol"]
    base = [x.double() for x in (Q, K, V)]
    for which in range(3):
        for _ in range(3):
            step = torch.randn(base[which].shape, dtype=torch.float64)
            eps = 1e-5
            moved = [[x + s * eps * step if k == which else x for k, x in enumerate(base)]
                     for s in (1, -1)]
            want = (loss(*moved[0]) - loss(*moved[1])) / (2 * eps)
            have = float((got[which] * step).sum())
            bound = float(((tol[which] + u * got[which].abs() + tiny(u)) * step.abs()).sum())
            assert abs(have - want) <= bound + 1e-6 * abs(want) + 1e-6


# ---- refusals of the binding ---------------------------------------------------------

def test_binding_refusals(gpu):
    cache = _cache(gpu, 4, 16, 2, 64)
    table, lens = torch.zeros((2, 2), dtype=torch.int32, device=DEV), _int32([3, 4])
    Q = torch.zeros((2, 1, 4, 64), dtype=torch.float16, device=DEV)
    K = torch.zeros((2, 1, 2, 64), dtype=torch.float16, device=DEV)
    attend = lambda *a, **k: gpu.cache_attend(cache, *a, **k)
    with pytest.raises(TypeError):
        attend(Q.float(), table, lens)
    with pytest.raises(TypeError):
        attend(Q.cpu(), table, lens)
    with pytest.raises(TypeError):
        attend(Q, table.long(), lens)
    with pytest.raises(TypeError):
        attend(Q, table, lens, prefix=table[0].long(), prefix_len=3)
    for bad in (Q[:1], Q[:, :, :3], Q[0], Q[..., :32], Q.transpose(1, 2),
                Q.expand(2, 2, 4, 64)):          # (both rows in one place)
        with pytest.raises(ValueError):
            attend(bad, table, lens)
    for kw in (dict(prefix=table[0]), dict(prefix_len=4), dict(prefix=table[0], prefix_len=33),
               dict(prefix=table, prefix_len=3), dict(prefix=table[0], prefix_len=-1),
               dict(out=torch.empty_like(Q)[:1]), dict(lse=torch.empty((2, 4), device=DEV)),
               dict(prefix=table[:, 0], prefix_len=3)):
        with pytest.raises(ValueError):
            attend(Q, table, lens, **kw)
    for t, m in ((table[0], lens), (table, lens[:1]), (table.t(), lens)):
        with pytest.raises(ValueError):
            gpu.cache_write(cache, K, K, t, m)
    with pytest.raises(TypeError):
        gpu.cache_write(cache, K, K.bfloat16(), table, lens)
    with pytest.raises(ValueError):
        gpu.cache_write(cache, K, K[:, :, :1], table, lens)
    with pytest.raises(TypeError):
        gpu.cache_read(cache, table, lens, 1, torch.int32)
    with pytest.raises(gpu.F3SError):
        attend(Q, table, lens, out=Q)
    with pytest.raises(gpu.F3SError):
        attend(Q, table, lens, scale=math.inf)
    codes = cache.k
    with pytest.raises(ValueError):
        gpu.Cache(codes, cache.v[:1], cache.k_exp, cache.v_exp)
    with pytest.raises(ValueError):
        gpu.Cache(codes.transpose(1, 2), cache.v, cache.k_exp, cache.v_exp)
    with pytest.raises(TypeError):
        gpu.Cache(codes.view(torch.uint8), cache.v, cache.k_exp, cache.v_exp)
    with pytest.raises(AttributeError):
        cache.k = cache.v                # (calls would go on reading the old place)
    odd = gpu.Cache.empty(2, 24, 1, 64)
    with pytest.raises(gpu.F3SError):
        gpu.cache_write(odd, K[:, :, :1].contiguous(), K[:, :, :1].contiguous(), table, lens)

    plan = gpu.CrossPlan([0, 3], [0, 5], 4, 2, 64)
    q = torch.zeros((3, 4, 64), dtype=torch.float16, device=DEV)
    k = torch.zeros((5, 2, 64), dtype=torch.float16, device=DEV)
    for a in ((q[:2], k, k), (q, k[:4], k), (q, q, k), (q.view(3, 256), k, k),
              (q, k, torch.zeros((2, 5, 64), dtype=torch.float16, device=DEV).transpose(0, 1))):
        with pytest.raises(ValueError):
            gpu.cross_forward(plan, *a)
    for a in ((q, k.bfloat16(), k), (q.float(), k, k), (q.cpu(), k, k)):
        with pytest.raises(TypeError):
            gpu.cross_forward(plan, *a)
    with pytest.raises(gpu.F3SError):
        gpu.cross_forward(plan, q, k, k, out=q)
    with pytest.raises(gpu.F3SError):
        gpu.cross_forward(plan, q, k, k, scale=math.nan)
    O, lse = gpu.cross_forward(plan, q, k, k)
    for a in ((O[:2], q, lse), (O, q[:2], lse), (O, q, lse[:2])):
        with pytest.raises(ValueError):
            gpu.cross_backward(plan, q, k, k, *a)
    with pytest.raises(TypeError):
        gpu.cross_backward(plan, q, k, k, O.float(), q, lse)
    for kw in (dict(heads=3, kv_heads=2), dict(heads=2, d=40), dict(heads=0)):
        with pytest.raises(gpu.F3SError):
            gpu.CrossPlan([0, 3], [0, 5], **{"kv_heads": 1, "d": 64, **kw})
    plan.close()
    with pytest.raises(RuntimeError):
        gpu.cross_forward(plan, q, k, k)
    plan.close()


# ---- streams, graphs, calls side by side ---------------------------------------------

def _decode_state(gpu, gen, B=5, n=2, kv=2, g=4, d=64, page=16, own=90, P=70):
    shared, each = -(-P // page), -(-own // page)
    cache = _cache(gpu, shared + B * each, page, kv, d)
    prefix = torch.arange(shared, dtype=torch.int32, device=DEV)
    table = (shared + torch.arange(B * each, dtype=torch.int32, device=DEV)).view(B, each)
    for pages, b, m in ((prefix.view(1, -1), 1, P), (table, B, own)):
        x = [_rows(gen, (b, m, kv, d), torch.bfloat16).to(DEV) for _ in "KV"]
        gpu.cache_write(cache, *x, pages, _int32([m] * b))
    Q = torch.randn((B, n, kv * g, d), generator=gen).to(torch.bfloat16).to(DEV)
    return cache, Q, table, prefix, P


def _capture(fn):
    side = torch.cuda.Stream(DEV)
    side.wait_stream(torch.cuda.current_stream(DEV))
    with torch.cuda.stream(side):
        fn()
    torch.cuda.current_stream(DEV).wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out = fn()
    torch.cuda.synchronize()
    return g, out


def test_graphs_with_changing_lengths(gpu, prefix_rows):
    """A captured step (write, attend) stays right while the lengths, which live
    on the device, grow and shrink; two graphs and eager work share the cache."""
    gen = torch.Generator().manual_seed(11)
    cache, Q, table, prefix, P = _decode_state(gpu, gen)
    B, n = Q.shape[:2]
    lens = _int32([90] * B)
    K, V = (_rows(gen, (B, n, 2, 64), torch.bfloat16).to(DEV) for _ in "KV")

    def step():
        gpu.cache_write(cache, K, V, table, lens)
        return gpu.cache_attend(cache, Q, table, lens, prefix=prefix, prefix_len=P)

    one, out1 = _capture(step)
    two, out2 = _capture(step)
    for r, now in enumerate(([1, 2, 3, 4, 5], [90, 0, 33, 64, 2], [16, 17, 31, 32, 92],
                             [90, 90, 1, 1, 50])):
        lens.copy_(_int32(now))
        K.copy_(torch.randn(K.shape, generator=gen).to(DEV))
        for x in out1 + out2:
            x.fill_(math.nan)
        torch.cuda.synchronize()
        one.replay()
        two.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        for out in (out1, out2):
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), r
        _compare(cache, Q.cpu(), table.cpu(), now, prefix, P, 0.125, *want)
        _ = (Q.float() * 2).sum().item()         # eager work between replays


def test_cross_graph_replays(gpu):
    gen = torch.Generator().manual_seed(12)
    plan = gpu.CrossPlan([0, 130, 170], [0, 700, 1500], 4, 2, 64)     # split both ways
    x = [torch.randn(s, generator=gen).half().to(DEV)
         for s in ((170, 4, 64), (1500, 2, 64), (1500, 2, 64), (170, 4, 64))]

    def step():
        O, lse = gpu.cross_forward(plan, *x[:3])
        return (O, lse) + gpu.cross_backward(plan, *x[:3], O, x[3], lse)

    graph, out = _capture(step)
    for r in range(3):
        for t in x:
            t.copy_(torch.randn(t.shape, generator=gen).half().to(DEV))
        for t in out:
            t.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), r
        assert all(bool(torch.isfinite(t).all()) for t in out)


def test_streams_and_calls_side_by_side(gpu, prefix_rows):
    """Calls on two other streams at once, on one plan and one cache, with tensors
    of their own streams: each as if alone, call after call."""
    gen = torch.Generator().manual_seed(13)
    cache, Q, table, prefix, P = _decode_state(gpu, gen, B=9)
    lens = _int32([5, 90, 33, 7, 64, 1, 80, 81, 16])
    plan = gpu.CrossPlan([0, 200, 230], [0, 900, 1400], 4, 1, 64)
    q = [torch.randn((230, 4, 64), generator=gen).half().to(DEV) for _ in range(2)]
    k = torch.randn((1400, 1, 64), generator=gen).half().to(DEV)
    want = [gpu.cross_forward(plan, x, k, k) for x in q]
    grads = [gpu.cross_backward(plan, x, k, k, w[0], x, w[1]) for x, w in zip(q, want)]
    base = gpu.cache_attend(cache, Q, table, lens, prefix=prefix, prefix_len=P)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(DEV) for _ in range(2)]
    got = []
    for _ in range(6):
        for s, x in zip(streams, q):
            O, lse = gpu.cross_forward(plan, x, k, k, stream=s)
            got.append((O, lse) + gpu.cross_backward(plan, x, k, k, O, x, lse, stream=s))
            got.append(gpu.cache_attend(cache, Q, table, lens, prefix=prefix, prefix_len=P,
                                        stream=s))
        with torch.cuda.stream(streams[0]):
            y = q[0] * 1                          # a tensor of that stream's own memory
            got.append(gpu.cross_forward(plan, y, k, k))
    torch.cuda.synchronize()
    for i in range(0, len(got), 5):
        for w, (cross, attend) in enumerate(((got[i], got[i + 1]), (got[i + 2], got[i + 3]))):
            for a, b in zip(cross, want[w] + grads[w]):
                assert torch.equal(a, b)
            assert torch.equal(attend[0], base[0]) and torch.equal(attend[1], base[1])
        assert torch.equal(got[i + 4][0], want[0][0])


def test_given_results(gpu):
    """Results in the caller's tensors; views at an offset as operands."""
    gen = torch.Generator().manual_seed(14)
    cache, Q, table, prefix, P = _decode_state(gpu, gen)
    lens = _int32([9, 90, 33, 7, 64])
    want = gpu.cache_attend(cache, Q, table, lens, prefix=prefix, prefix_len=P)
    room = torch.full((7,) + Q.shape[1:], math.nan, dtype=Q.dtype, device=DEV)
    stats = torch.full((7,) + Q.shape[1:3], math.nan, device=DEV)
    out = gpu.cache_attend(cache, torch.cat([Q[:1], Q])[1:], table, lens, prefix=prefix,
                           prefix_len=P, out=room[1:6], lse=stats[1:6])
    assert out[0].data_ptr() == room[1:6].data_ptr()
    assert torch.equal(room[1:6], want[0]) and torch.equal(stats[1:6], want[1])
    assert bool(room[[0, 6]].isnan().all()) and bool(stats[[0, 6]].isnan().all())
    plan = gpu.CrossPlan([0, 3, 7], [0, 40, 70], 8, 2, 64)
    q, k = torch.randn((9, 8, 64), device=DEV).half(), torch.randn((72, 2, 64), device=DEV).half()
    O = torch.full((9, 8, 64), math.nan, dtype=torch.float16, device=DEV)
    lse = torch.full((9, 8), math.nan, device=DEV)
    gpu.cross_forward(plan, q[1:8], k[1:71], k[2:72], out=O[1:8], lse=lse[1:8])
    want = gpu.cross_forward(plan, q[1:8].clone(), k[1:71].clone(), k[2:72].clone())
    assert torch.equal(O[1:8], want[0]) and torch.equal(lse[1:8], want[1])
    assert bool(O[[0, 8]].isnan().all()) and bool(lse[[0, 8]].isnan().all())


# ---- sizes -----------------------------------------------------------------------------

def test_rows_beyond_4_gib(gpu):
    """Keys and pages whose offsets pass 32 bits."""
    kv, d = 8, 128
    first = (1 << 32) // (kv * d * 2) + 77
    K, V = (torch.randn((first + 300, kv, d), device=DEV).to(torch.bfloat16) for _ in "KV")
    Q = torch.randn((140, 16, d), device=DEV).to(torch.bfloat16)
    plan = gpu.CrossPlan([0, 0, 140], [0, first, first + 300], 16, kv, d)
    small = gpu.CrossPlan([0, 140], [0, 300], 16, kv, d)
    O, lse = gpu.cross_forward(plan, Q, K, V)
    tail = K[first:].clone(), V[first:].clone()
    want = gpu.cross_forward(small, Q, *tail)
    assert torch.equal(O, want[0]) and torch.equal(lse, want[1])
    got = gpu.cross_backward(plan, Q, K, V, O, Q, lse)
    grads = gpu.cross_backward(small, Q, *tail, O, Q, lse)
    assert torch.equal(got[0], grads[0])
    for a, b in zip(got[1:], grads[1:]):
        assert torch.equal(a[first:], b)
        assert not a[:first:1000].any()
    del K, V, got
    pages = (1 << 32) // (256 * kv * d) + 9
    cache = gpu.Cache.empty(pages, 256, kv, d)
    near = gpu.Cache.empty(8, 256, kv, d)
    x = [torch.randn((2, 700, kv, d), device=DEV).to(torch.bfloat16) for _ in "KV"]
    lens = _int32([700, 555])
    far_table = _int32([[pages - 1, pages - 3, pages - 5], [pages - 2, 3, pages - 4]])
    near_table = _int32([[7, 5, 3], [6, 0, 4]])
    q = torch.randn((2, 1, 16, d), device=DEV).to(torch.bfloat16)
    results = []
    for c, t in ((cache, far_table), (near, near_table)):
        gpu.cache_write(c, *x, t, lens)
        results.append(gpu.cache_attend(c, q, t, lens, prefix=t[0], prefix_len=300)
                       + gpu.cache_read(c, t, lens, 700, torch.bfloat16))
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B,n,lens", [(1, 130, [130]), (2, 70, [200, 75]), (300, 1, None),
                                      (70, 2, None)])
def test_many_new_tokens_and_many_sequences(gpu, B, n, lens):
    lens = [(37 * b) % 90 for b in range(B)] if lens is None else lens
    _attend_case(gpu, torch.float16, 32, 32, 1, 2, lens, n, 21)


def test_thousands_of_sequences(gpu):
    """More sequences than a wave looks at in one go: every one as if alone."""
    gen = torch.Generator().manual_seed(31)
    kv, d, page, B = 2, 64, 16, 5000
    table7, n_pages = _table(gen, 7, 60)         # (room for more: found on the device)
    cache = _cache(gpu, n_pages, page, kv, d)
    x = [_rows(gen, (7, 64, kv, d), torch.float16).to(DEV) for _ in "KV"]
    gpu.cache_write(cache, *x, table7.to(DEV), _int32([64] * 7))
    lens7 = [0, 1, 63, 64, 17, 40, 33]
    Q7 = torch.randn((7, 1, 4, d), generator=gen).half()
    pick = torch.randint(0, 7, (B,), generator=gen)
    lens = torch.tensor(lens7)[pick]
    O, lse = gpu.cache_attend(cache, Q7[pick].to(DEV), table7[pick].to(DEV),
                              lens.to(torch.int32).to(DEV))
    first = [int((pick == k).nonzero()[0]) for k in range(7)]
    _compare(cache, Q7, table7, lens7, None, 0, 0.125, O[first], lse[first])
    # (a sequence this short is one piece wherever it stands)
    at = torch.tensor(first)[pick].to(DEV)
    assert torch.equal(O, O[at]) and torch.equal(lse, lse[at])
    # the same keys as one plan's: sequences of one token over 0 .. 64 rows
    plan = gpu.CrossPlan(range(B + 1), _sums(lens.tolist()), 4, kv, d)
    K, V = (torch.cat([x[w][int(k), :lens7[int(k)]] for k in pick]) for w in range(2))
    C, clse = gpu.cross_forward(plan, Q7[pick].to(DEV).view(B, 4, d), K, V)
    assert torch.equal(C, C[at]) and torch.equal(clse, clse[at])
    G = torch.randn((7, 4, d), generator=gen).half()[pick].to(DEV)
    grads = gpu.cross_backward(plan, Q7[pick].to(DEV).view(B, 4, d), K, V, C, G, clse)
    assert torch.equal(grads[0], grads[0][at])
    for got in grads[1:]:
        assert bool(torch.isfinite(got).all())


# ---- all of it together -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
def test_a_decoder_generates(gpu, dtype):
    """A decoder layer behind a long shared prompt: ragged prompts enter the cache
    (padded on the left), then tokens one by one, each attending to the prompt,
    to the cache and to its encoder's states; every step against 64 bits."""
    gen = torch.Generator().manual_seed(21)
    B, kv, g, d, page, P = 4, 2, 3, 64, 32, 131
    H, own = kv * g, [9, 1, 40, 33]
    steps, each, shared = 4, 3, 5
    cache = _cache(gpu, shared + B * each, page, kv, d)
    prefix = torch.tensor([3, 0, 4, 1, 2], dtype=torch.int32, device=DEV)
    table = (shared + torch.randperm(B * each, generator=gen)).to(torch.int32).view(B, each)
    new = lambda *s: torch.randn(s, generator=gen).to(dtype).to(DEV)
    gpu.cache_write(cache, new(1, P, kv, d), new(1, P, kv, d), prefix.view(1, -1), _int32([P]))
    states = [17, 300, 1, 64]
    k_ptr = _sums(states)
    EK, EV = new(k_ptr[-1], kv, d), new(k_ptr[-1], kv, d)
    plan = gpu.CrossPlan(list(range(B + 1)), k_ptr, H, kv, d)
    top = max(own)
    gpu.cache_write(cache, new(B, top, kv, d), new(B, top, kv, d), table.to(DEV), _int32(own))
    Q = new(B, top, H, d)
    O, lse = gpu.cache_attend(cache, Q, table.to(DEV), _int32(own), prefix=prefix, prefix_len=P)
    _compare(cache, Q.cpu(), table, own, prefix, P, 0.125, O, lse)
    lens, u = _int32(own), half_step(dtype)
    for t in range(1, steps + 1):
        lens += 1
        now = [m + t for m in own]
        gpu.cache_write(cache, new(B, 1, kv, d), new(B, 1, kv, d), table.to(DEV), lens)
        Q = new(B, 1, H, d)
        O, lse = gpu.cache_attend(cache, Q, table.to(DEV), lens, prefix=prefix, prefix_len=P)
        _compare(cache, Q.cpu(), table, now, prefix, P, 0.125, O, lse)
        q = (Q + O).view(B, H, d)                 # the residual feeds the next operator
        C, clse = gpu.cross_forward(plan, q, EK, EV)
        for b in range(B):
            j = slice(k_ptr[b], k_ptr[b + 1])
            for h in range(H):
                f = attention(q[b: b + 1, h].double().cpu(), EK[j, h // g].double().cpu(),
                              EV[j, h // g].double().cpu(), 0.125, u)
                close(C[b: b + 1, h], f["O"], f["O_tol"], ("cross", t, b, h))
                close(clse[b: b + 1, h], f["lse"], f["lse_tol"], ("lse", t, b, h))


# ---- failures ------------------------------------------------------------------------------

def test_a_plan_out_of_memory(gpu, monkeypatch):
    """No room for a plan's lists is an error that the next plan does not feel."""
    monkeypatch.setenv("F3S_ALLOC_LIMIT_BYTES", "64")
    with pytest.raises(gpu.F3SError, match="OUT_OF_MEMORY"):
        gpu.CrossPlan([0, 300], [0, 300], 4, 2, 64)
    monkeypatch.delenv("F3S_ALLOC_LIMIT_BYTES")
    _case(gpu, torch.float16, 64, 2, 2, [30, 3], [70, 33])
