"""Cross attention whose passes are divided into pieces, against plain 64-bit
attention and gradients: partial results of dK and dV, of dQ and of the forward
by full and ragged tiles, and the batches whose last tiles alone are divided."""
import math

import pytest
import torch

from _dense import F32, attention, close, gradients, half_step, tiny

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
TYPES = [torch.float16, torch.bfloat16]


def _round256(n):
    return -(-n // 256) * 256


def _parts(plan):
    """Bytes of partial sums that a backward of the plan keeps."""
    return plan._backward_bytes - _round256(plan.q_shape[0] * plan.heads * 8)


def _case(gpu, dtype, d, kv, g, q_len, k_len, padded=False):
    gen = torch.Generator().manual_seed(d + kv + sum(q_len))
    H, B = kv * g, len(q_len)
    room = [q + 3 if padded else q for q in q_len], [k + 5 if padded else k for k in k_len]
    q_ptr, k_ptr = ([sum(x[:b]) for b in range(B + 1)] for x in room)
    Q, G = (torch.randn((q_ptr[-1], H, d), generator=gen).to(dtype) for _ in "QG")
    K, V = (torch.randn((k_ptr[-1], kv, d), generator=gen).to(dtype) for _ in "KV")
    for x, ptr, n in ((Q, q_ptr, q_len), (G, q_ptr, q_len), (K, k_ptr, k_len), (V, k_ptr, k_len)):
        for b in range(B):
            x[ptr[b] + n[b]: ptr[b + 1]] = math.nan
    plan = gpu.CrossPlan(q_ptr, k_ptr, H, kv, d, q_len=q_len if padded else None,
                         k_len=k_len if padded else None, device=DEV)
    Q, K, V, G = dev = [x.to(DEV) for x in (Q, K, V, G)]
    O, lse = gpu.cross_forward(plan, Q, K, V)
    got = dict(zip(("dQ", "dK", "dV"), gpu.cross_backward(plan, Q, K, V, O, G, lse)), O=O,
               lse=lse)
    u, scale = half_step(dtype), 1 / math.sqrt(d)
    want = {n: torch.zeros(got[n].shape, dtype=torch.float64, device=DEV) for n in got}
    tol = {n: torch.zeros_like(x) for n, x in want.items()}
    want["lse"].fill_(-math.inf)
    for b in range(B):
        i = slice(q_ptr[b], q_ptr[b] + q_len[b])
        j = slice(k_ptr[b], k_ptr[b] + k_len[b])
        for h in range(H):
            q, k, v, w = (x.double() for x in (Q[i, h], K[j, h // g], V[j, h // g], G[i, h]))
            f = attention(q, k, v, scale, u)
            r = gradients(q, k, v, w, scale, u, f)
            for n in ("O", "lse"):
                want[n][i, h], tol[n][i, h] = f[n], f[n + "_tol"]
            want["dQ"][i, h], tol["dQ"][i, h] = r["dQ"], r["dQ_tol"]
            # (a running sum goes over the rows of all heads of the group)
            more = (g * q_len[b] / 16 + 64) * F32
            dS = (f["P"] * (w @ v.T - (w * f["O"]).sum(1, keepdim=True))).abs()
            tol["dV"][j, h // g] += more * (f["P"].T @ w.abs())
            tol["dK"][j, h // g] += more * scale * (dS.T @ q.abs())
            for n in ("dK", "dV"):
                want[n][j, h // g] += r[n]
                tol[n][j, h // g] += r[n + "_tol"]
    for n in ("dQ", "dK", "dV"):
        tol[n] += u * want[n].abs() + tiny(u)
    for n in want:
        close(got[n], want[n].cpu(), tol[n].cpu(), n)
    return plan


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("d,kv,g,q,k", [
    (64, 2, 4, [400], [300]), (128, 1, 8, [300], [400]), (96, 1, 3, [700], [333]),
    (160, 1, 2, [900], [300]), (256, 1, 1, [2000], [130]), (32, 1, 4, [1000], [200]),
    (224, 2, 2, [1100, 40], [200, 33]), (192, 1, 4, [600, 300], [70, 257]),
])
def test_divided_keys(gpu, dtype, padded, d, kv, g, q, k):
    """dK and dV of many query rows and few keys: in pieces.  (448 keys and fewer
    are never divided, so that what a backward keeps are dK's and dV's.)"""
    plan = _case(gpu, dtype, d, kv, g, q, k, padded)
    assert max(k) <= 448 and plan._forward_bytes == 0
    assert _parts(plan) >= 2 * 2 * 4 * d * kv * max(k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("d,kv,g,q,k", [
    (64, 1, 1, [33, 100], [2000, 1500]), (128, 2, 1, [120], [3000]), (96, 2, 1, [65], [1000]),
    (160, 1, 1, [128], [2000]), (256, 1, 1, [127], [2000]), (32, 1, 2, [97], [1500]),
    (192, 1, 2, [48, 10], [700, 900]), (224, 1, 4, [32], [1200]),
])
def test_divided_queries(gpu, monkeypatch, dtype, padded, d, kv, g, q, k):
    """The forward and dQ by the kernels of 128 rows, few tiles over many keys: in
    pieces, with one to four waves that have rows.  (Nor are 448 query rows.)"""
    monkeypatch.setenv("F3S_CROSS_ROWS", "128")
    plan = _case(gpu, dtype, d, kv, g, q, k, padded)
    assert g * max(q) <= 448
    assert plan._forward_bytes >= 2 * 4 * d * kv * g * max(q)
    assert _parts(plan) >= 2 * 4 * d * kv * g * max(q)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,q,k", [(256, 8202, 2000), (256, 2000, 4106), (160, 2000, 4106)])
def test_divided_tails(gpu, monkeypatch, dtype, d, q, k):
    """A few tiles too many for a round (260 on 256 places, 132 on 128): the last 10
    rows of each of the 4 heads alone are divided, on one side of the batch."""
    monkeypatch.setenv("F3S_CROSS_ROWS", "128")
    plan = _case(gpu, dtype, d, 4, 1, [q], [k])
    if q > k:
        assert 0 < plan._forward_bytes < 4 * q * d * 4          # (not all rows, even once)
    else:
        # (dQ is divided as the forward is, whose partial rows have 8 bytes more)
        rest = _parts(plan) - plan._forward_bytes * d // (d + 2)
        assert 1024 < rest < 4 * k * 2 * d * 4
