"""Causal attention with a sliding window and sinks on the GPU against plain 64-bit
attention and gradients."""
import math

import pytest
import torch

from _dense import attention, close, gradients, half_step, tiny

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
TYPES = [torch.float16, torch.bfloat16]


def _sums(x):
    out = [0]
    for v in x:
        out.append(out[-1] + v)
    return out


def seen_keys(nq, nk, window, sinks):
    """[nq, nk]: which keys each of the newest nq tokens sees."""
    p = torch.arange(nk - nq, nk)[:, None]
    j = torch.arange(nk)
    return (j <= p) & ((p - j < (nk if window is None else window)) | (j < sinks))


def _case(gpu, dtype, d, kv, g, q_len, k_len, window, sinks, padded=False, scale=None,
          grad=True, seed=0, tweak=None):
    gen = torch.Generator().manual_seed(seed + d + kv + len(q_len) + sum(q_len))
    H, B = kv * g, len(q_len)
    q_ptr, k_ptr = _sums(q_len), _sums(k_len)
    if padded:
        q_ptr = [(max(q_len) + 1) * b for b in range(B + 1)]
        k_ptr = [(max(k_len) + 2) * b for b in range(B + 1)]
    scale = 1 / math.sqrt(d) if scale is None else scale
    Q, G = (torch.randn((q_ptr[-1], H, d), generator=gen).to(dtype) for _ in "QG")
    K, V = (torch.randn((k_ptr[-1], kv, d), generator=gen).to(dtype) for _ in "KV")
    if tweak:
        tweak(Q, K, V, G)
    q_pad, k_pad = (torch.ones(p[-1], dtype=torch.bool) for p in (q_ptr, k_ptr))
    for b in range(B):
        q_pad[q_ptr[b]: q_ptr[b] + q_len[b]] = False
        k_pad[k_ptr[b]: k_ptr[b] + k_len[b]] = False
    for x, pad in ((Q, q_pad), (G, q_pad), (K, k_pad), (V, k_pad)):
        x[pad] = math.nan                   # what padding holds does not matter
    plan = gpu.WindowPlan(q_ptr, k_ptr, H, kv, d, window=window, sinks=sinks,
                          q_len=q_len if padded else None, k_len=k_len if padded else None,
                          device=DEV)
    dev = [x.to(DEV) for x in (Q, K, V, G)]
    O, lse = gpu.window_forward(plan, *dev[:3], scale=scale)
    grads = gpu.window_backward(plan, *dev[:3], O, dev[3], lse, scale=scale) if grad else None
    torch.cuda.synchronize()

    u = half_step(dtype)
    want = {n: torch.zeros(Q.shape, dtype=torch.float64) for n in ("O", "dQ")}
    want.update({n: torch.zeros(K.shape, dtype=torch.float64) for n in ("dK", "dV")})
    tol = {n: torch.zeros_like(x) for n, x in want.items()}
    want["lse"] = torch.full(Q.shape[:2], -math.inf, dtype=torch.float64)
    tol["lse"] = torch.zeros_like(want["lse"])
    for b in range(B):
        i = slice(q_ptr[b], q_ptr[b] + q_len[b])
        j = slice(k_ptr[b], k_ptr[b] + k_len[b])
        seen = seen_keys(q_len[b], k_len[b], window, sinks)
        for h in range(H):
            q, k, v, w = (x.double() for x in (Q[i, h], K[j, h // g], V[j, h // g], G[i, h]))
            f = attention(q, k, v, scale, u, seen=seen)
            for n in ("O", "lse"):
                want[n][i, h], tol[n][i, h] = f[n], f[n + "_tol"]
            if grad:
                r = gradients(q, k, v, w, scale, u, f)
                want["dQ"][i, h], tol["dQ"][i, h] = r["dQ"], r["dQ_tol"]
                for n in ("dK", "dV"):
                    want[n][j, h // g] += r[n]
                    tol[n][j, h // g] += r[n + "_tol"]
    close(O, want["O"], tol["O"], "O")
    close(lse, want["lse"], tol["lse"], "lse")
    if grad:
        for n, x in zip(("dQ", "dK", "dV"), grads):
            close(x, want[n], tol[n] + u * want[n].abs() + tiny(u), n)
    return plan, dev, O, lse, grads


# d, key heads, query heads of each, query and key rows, window, sinks
CASES = [
    (64, 2, 1, [1, 5, 33, 0], [1, 5, 33, 7], 8, 0),
    (64, 1, 4, [3, 20, 100], [3, 20, 100], 1, 0),
    (64, 1, 2, [150, 129], [150, 129], 40, 3),
    (128, 2, 4, [1, 1], [500, 301], 64, 4),
    (128, 1, 2, [130, 5], [400, 64], 100, 65),
    (128, 1, 5, [77], [77], None, 0),
    (128, 1, 1, [300], [300], 128, 0),
    (32, 3, 1, [40, 0, 17], [31, 20, 0], 9, 2),        # more queries than keys
    (96, 1, 3, [170], [170], 64, 64),
    (256, 1, 1, [133, 64], [133, 200], 50, 1),
    (160, 1, 2, [120], [140], 33, 0), (192, 1, 1, [65], [333], 1000, 5),
    (224, 1, 1, [90], [130], 31, 31),
    (64, 1, 1, [300, 257], [513, 257], 256, 200),
    (64, 2, 2, [40], [40], 0, 0), (64, 1, 2, [140], [200], 0, 5),   # nothing; sinks alone
    (64, 1, 8, [260], [260], 17, 130),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("d,kv,g,q,k,window,sinks", CASES)
def test_forward_and_gradients(gpu, dtype, padded, d, kv, g, q, k, window, sinks):
    _case(gpu, dtype, d, kv, g, q, k, window, sinks, padded=padded)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,kv,g,n,window,sinks", [
    (64, 1, 2, 2500, None, 0),      # the longest walks are divided
    (64, 1, 4, 1800, 200, 4),       # the sinks' walk is
    (128, 1, 1, 1500, 700, 130),
    (256, 1, 1, 900, 500, 2),
])
def test_divided(gpu, dtype, d, kv, g, n, window, sinks):
    plan = _case(gpu, dtype, d, kv, g, [n], [n], window, sinks, seed=2)[0]
    assert plan._forward_bytes > 0 or plan._backward_bytes > 8 * n * kv * g + 256


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(gpu, dtype, scale):
    _case(gpu, dtype, 64, 1, 2, [90], [120], 30, 2, scale=scale)


@pytest.mark.parametrize("large", [60000.0, 250.0])
def test_what_lies_outside_the_window_has_no_part(gpu, large):
    """Rows that a token does not see may hold anything finite, and change no bit of its
    result: not those of its tile either."""
    n, window, sinks = 700, 90, 3
    gen = torch.Generator().manual_seed(5)
    Q, K, V = (torch.randn((n, 2, 64), generator=gen).half().to(DEV) for _ in "QKV")
    plan = gpu.WindowPlan([0, n], [0, n], 2, 2, 64, window=window, sinks=sinks, device=DEV)
    O, lse = gpu.window_forward(plan, Q, K, V)
    t = 400
    K2, V2 = K.clone(), V.clone()
    for x in (K2, V2):
        x[t + 1:] = -large
        x[sinks: t - window + 1] = large
    O2, lse2 = gpu.window_forward(plan, Q, K2, V2)
    assert torch.equal(O[t], O2[t]) and torch.equal(lse[t], lse2[t])


def test_a_long_window_is_causal_attention(gpu):
    """As one query row over all keys, and with sinks that change nothing."""
    n = 333
    gen = torch.Generator().manual_seed(6)
    Q, K, V = (torch.randn((n, 1, 64), generator=gen).half().to(DEV) for _ in "QKV")
    whole = gpu.WindowPlan([0, n], [0, n], 1, 1, 64, device=DEV)
    O, lse = gpu.window_forward(whole, Q, K, V)
    for more in (dict(window=n), dict(window=n, sinks=7), dict(window=5, sinks=n),
                 dict(window=2**31 - 1, sinks=2**31 - 1)):
        plan = gpu.WindowPlan([0, n], [0, n], 1, 1, 64, device=DEV, **more)
        O2, lse2 = gpu.window_forward(plan, Q, K, V)
        assert torch.equal(O, O2) and torch.equal(lse, lse2)
    last = gpu.CrossPlan([0, 1], [0, n], 1, 1, 64, device=DEV)
    O3, lse3 = gpu.cross_forward(last, Q[-1:], K, V)
    assert torch.allclose(O3.float(), O[-1:].float(), atol=2e-3)
    assert torch.allclose(lse3, lse[-1:], atol=1e-5)


def test_differences(gpu):
    """Gradients against central differences of the forward, in the direction of the
    gradient (fp16 operands, a step that they hold exactly)."""
    n, window, sinks, d = 60, 20, 2, 64
    gen = torch.Generator().manual_seed(7)
    Q, K, V, G = ((torch.randn((n, 2, d), generator=gen)).half() for _ in "QKVG")
    f = attention  # the 64-bit forward
    scale = 1 / 8
    seen = seen_keys(n, n, window, sinks)
    plan = gpu.WindowPlan([0, n], [0, n], 2, 2, d, window=window, sinks=sinks, device=DEV)
    dev = [x.to(DEV) for x in (Q, K, V)]
    O, lse = gpu.window_forward(plan, *dev)
    grads = gpu.window_backward(plan, *dev, O, G.to(DEV), lse)

    def loss(x):
        return sum(float((f(*(y[:, h] for y in x), scale, 0.0, seen=seen)["O"]
                          * G[:, h].double()).sum()) for h in range(2))

    at = [x.double() for x in (Q, K, V)]
    for k, grad in enumerate(grads):
        way = grad.double().cpu()
        way = way / way.norm()
        e = 1e-4
        up = [x + e * way * (i == k) for i, x in enumerate(at)]
        down = [x - e * way * (i == k) for i, x in enumerate(at)]
        slope = (loss(up) - loss(down)) / (2 * e)
        # the gradient's own length, off by its 16-bit roundings (three of 2^-11 each)
        assert abs(slope - float(grad.double().norm())) < 3 * 2.0 ** -11 * slope


def test_captured(gpu):
    """Forward and backward in a graph, replayed with other inputs, while the plan's
    eager calls run in between."""
    n = 500
    plan = gpu.WindowPlan([0, 200, n], [0, 200, n], 4, 2, 64, window=70, sinks=4, device=DEV)
    Q, G = (torch.zeros((n, 4, 64), dtype=torch.float16, device=DEV) for _ in "QG")
    K, V = (torch.zeros((n, 2, 64), dtype=torch.float16, device=DEV) for _ in "KV")

    def step():
        O, lse = gpu.window_forward(plan, Q, K, V)
        return (O, lse) + gpu.window_backward(plan, Q, K, V, O, G, lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        for x in (Q, K, V, G):
            x.copy_(torch.randn(x.shape, generator=gen, device=DEV))
        eager = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


def test_streams_and_refusals(gpu):
    n = 100
    plan = gpu.WindowPlan([0, n], [0, n], 2, 1, 64, window=16, device=DEV)
    cross = gpu.CrossPlan([0, n], [0, n], 2, 1, 64, device=DEV)
    Q = torch.randn((n, 2, 64), device=DEV).half()
    K, V = (torch.randn((n, 1, 64), device=DEV).half() for _ in "KV")
    O, lse = gpu.window_forward(plan, Q, K, V)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    O2, lse2 = gpu.window_forward(plan, Q, K, V, stream=other)
    other.synchronize()
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    with pytest.raises(TypeError):
        gpu.window_forward(cross, Q, K, V)
    with pytest.raises(TypeError):
        gpu.cross_forward(plan, Q, K, V)
    with pytest.raises(TypeError):
        gpu.window_backward(cross, Q, K, V, O, O, lse)
    with pytest.raises(ValueError):
        gpu.window_forward(plan, Q[1:], K, V)
    with pytest.raises(TypeError):
        gpu.window_forward(plan, Q, K.float(), V)
    with pytest.raises(ValueError):
        gpu.window_forward(plan, Q.transpose(0, 1), K, V)
    with pytest.raises(gpu.F3SError):
        gpu.window_forward(plan, Q, K, V, out=Q)
    plan.close()
    with pytest.raises(RuntimeError):
        gpu.window_forward(plan, Q, K, V)
