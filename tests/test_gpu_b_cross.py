"""Cross attention on the GPU against plain 64-bit attention and gradients."""
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


def _case(gpu, dtype, d, kv, g, q_len, k_len, padded=False, scale=None, grad=True, seed=0):
    gen = torch.Generator().manual_seed(seed + d + kv + len(q_len) + sum(q_len))
    H, B = kv * g, len(q_len)
    q_ptr, k_ptr = _sums(q_len), _sums(k_len)
    if padded:
        q_ptr = [(max(q_len) + 1) * b for b in range(B + 1)]
        k_ptr = [(max(k_len) + 2) * b for b in range(B + 1)]
    scale = 1 / math.sqrt(d) if scale is None else scale
    Q, G = (torch.randn((q_ptr[-1], H, d), generator=gen).to(dtype) for _ in "QG")
    K, V = (torch.randn((k_ptr[-1], kv, d), generator=gen).to(dtype) for _ in "KV")
    q_pad, k_pad = (torch.ones(p[-1], dtype=torch.bool) for p in (q_ptr, k_ptr))
    for b in range(B):
        q_pad[q_ptr[b]: q_ptr[b] + q_len[b]] = False
        k_pad[k_ptr[b]: k_ptr[b] + k_len[b]] = False
    for x, pad in ((Q, q_pad), (G, q_pad), (K, k_pad), (V, k_pad)):
        x[pad] = math.nan                   # what padding holds does not matter
    plan = gpu.CrossPlan(q_ptr, k_ptr, H, kv, d, q_len=q_len if padded else None,
                         k_len=k_len if padded else None, device=DEV)
    dev = [x.to(DEV) for x in (Q, K, V, G)]
    O, lse = gpu.cross_forward(plan, *dev[:3], scale=scale)
    grads = gpu.cross_backward(plan, *dev[:3], O, dev[3], lse, scale=scale) if grad else None
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
        for h in range(H):
            q, k, v, w = (x.double() for x in (Q[i, h], K[j, h // g], V[j, h // g], G[i, h]))
            f = attention(q, k, v, scale, u)
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


CASES = [
    (64, 2, 1, [1, 1, 1], [5, 33, 0]),
    (64, 1, 4, [3, 20, 1], [64, 1, 100]),
    (128, 2, 4, [1, 1], [1000, 301]),
    (128, 1, 2, [130, 5], [129, 64]),
    (32, 3, 1, [40, 0, 17], [31, 20, 0]),
    (96, 1, 3, [70], [65]),
    (256, 1, 1, [33, 64], [70, 200]),
    (160, 1, 2, [12], [40]), (192, 1, 1, [65], [33]), (224, 1, 1, [9], [130]),
    (64, 1, 1, [300, 257], [513, 100]),
]


@pytest.mark.parametrize("rows", ["16", "128"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("d,kv,g,q,k", CASES)
def test_forward(gpu, monkeypatch, rows, dtype, padded, d, kv, g, q, k):
    """By the kernel of 16 query rows and by that of 128."""
    monkeypatch.setenv("F3S_CROSS_ROWS", rows)
    _case(gpu, dtype, d, kv, g, q, k, padded=padded, grad=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("d,kv,g,q,k", CASES)
def test_gradients(gpu, dtype, padded, d, kv, g, q, k):
    _case(gpu, dtype, d, kv, g, q, k, padded=padded, seed=1)
