"""Values of the dense operators where 16 bits of a product's operands could lose
them: tokens before one whose values are far larger, probabilities of very many
keys."""
import math

import pytest
import torch

from _dense import F32, attention, close, half_step
from test_gpu_b_cache import TYPES, _cache, _rows, _table, _values

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---- what a token does not see ------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,page,kv,g,lens,n,P,room", [
    (64, 16, 1, 2, [40, 9, 4], 4, 0, 0),          # one workgroup has all keys
    (64, 32, 2, 1, [70, 33], 9, 0, 3000),         # several, and a join
    (128, 16, 1, 4, [33, 1, 130], 5, 40, 3000),   # behind a prefix
    (256, 64, 1, 3, [65, 64], 2, 0, 0),
    (32, 16, 1, 1, [50], 40, 0, 0),               # rows of several blocks
])
def test_later_tokens_with_large_values(gpu, dtype, d, page, kv, g, lens, n, P, room):
    """The newest token's values are 2^24 (fp16) or 2^60 (bf16) times the others': the
    tokens before it, which do not see them, lose no bits, and are what they are
    behind an ordinary token, bit by bit."""
    gen = torch.Generator().manual_seed(d + n)
    B, shared = len(lens), -(-P // page)
    table, n_pages = _table(gen, B, -(-max(max(lens), room) // page), first=shared)
    cache = _cache(gpu, n_pages, page, kv, d)
    prefix = torch.arange(shared, dtype=torch.int32) if P else None
    at = {} if prefix is None else dict(prefix=prefix.to(DEV), prefix_len=P)
    small, large = (2.0 ** -10, 2.0 ** 14) if dtype is torch.float16 else (1.0, 2.0 ** 60)
    if P:
        x = [_rows(gen, (1, P, kv, d), torch.float32).clamp(-3, 3).to(dtype) for _ in "KV"]
        gpu.cache_write(cache, x[0].to(DEV), (x[1] * small).to(DEV), prefix.view(1, -1).to(DEV),
                        _int32([P]))
    top = max(lens)
    K, V = (_rows(gen, (B, top, kv, d), torch.float32).clamp(-3, 3) for _ in "KV")
    Q = torch.randn((B, n, kv * g, d), generator=gen).to(dtype)
    results = []
    for size in (small, large):
        V2 = torch.cat([V[:, :-1] * small, V[:, -1:] * size], 1)
        gpu.cache_write(cache, K.to(dtype).to(DEV), V2.to(dtype).to(DEV), table.to(DEV),
                        _int32(lens))
        results.append(gpu.cache_attend(cache, Q.to(DEV), table.to(DEV), _int32(lens), **at))
    (O1, lse1), (O, lse) = results
    # (sequences of one token: the last)
    assert torch.equal(O[:, :-1], O1[:, :-1]) and torch.equal(lse, lse1)
    values = _values(cache)
    for b, m in enumerate(lens):
        pos = torch.arange(m)
        k, v = (x[table[b][pos // page].long(), :, pos % page] for x in values)
        if P:
            pp = torch.arange(P)
            k, v = (torch.cat([x[prefix[pp // page].long(), :, pp % page], y])
                    for x, y in zip(values, (k, v)))
        for t in range(n):
            see = P + max(0, m - n + 1 + t)
            for h in range(kv * g):
                x, y = k[:see, h // g], v[:see, h // g]
                # (a probability too small for f16: 2^-25 of the largest value seen)
                floor = torch.full((see, 1), 2.0 ** -25) * (y.abs().max() if see else 0.0)
                f = attention(Q[b, t: t + 1, h].double(), x, y, 1 / math.sqrt(d),
                              half_step(dtype), up=2.0 ** -11, floor=2 * floor)
                # (without the bound of f16 values next to 0 for a seen row: its
                # probabilities are relative to its own largest power)
                close(O[b, t: t + 1, h], f["O"], f["O_tol"], (b, t, h))
                close(lse[b, t: t + 1, h], f["lse"], f["lse_tol"], ("lse", b, t, h))


# ---- probabilities of very many keys ---------------------------------------------------

@pytest.mark.parametrize("d,kv,g,q_len,k_len", [
    (32, 1, 1, [1, 3], [360000, 30000]), (64, 1, 2, [1], [130500]), (160, 1, 1, [2], [200100]),
    (128, 2, 2, [2], [50123]), (32, 1, 1, [400], [40001]),       # (divided: many query rows)
])
def test_value_gradients_of_many_keys(gpu, d, kv, g, q_len, k_len):
    """dV in fp16 where every probability is far below 2^-14, fp16's least normal
    number: each keeps its 11 bits all the same.  (dO is as large as a scaled loss
    makes it, so that dV itself is a normal number.)"""
    gen = torch.Generator().manual_seed(d + kv + g)
    dtype, u, H, scale = torch.float16, 2.0 ** -11, kv * g, 1 / math.sqrt(d)
    q_ptr, k_ptr = ([sum(x[:b]) for b in range(len(x) + 1)] for x in (q_len, k_len))
    Q = (torch.randn((q_ptr[-1], H, d), generator=gen) / 1024).to(dtype).to(DEV)
    G = (torch.randn((q_ptr[-1], H, d), generator=gen) * 512).to(dtype).to(DEV)
    K, V = (torch.randn((k_ptr[-1], kv, d), generator=gen).to(dtype).to(DEV) for _ in "KV")
    plan = gpu.CrossPlan(q_ptr, k_ptr, H, kv, d, device=DEV)
    O, lse = gpu.cross_forward(plan, Q, K, V)
    got = gpu.cross_backward(plan, Q, K, V, O, G, lse)[2]
    want = torch.zeros(V.shape, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(want)
    for b in range(len(q_len)):
        i, j = slice(q_ptr[b], q_ptr[b + 1]), slice(k_ptr[b], k_ptr[b + 1])
        for h in range(H):
            q, k, w = Q[i, h].double(), K[j, h // g].double(), G[i, h].double()
            x = q @ k.T * scale
            lse64 = torch.logsumexp(x, 1, keepdim=True)
            P = torch.exp(x - lse64)
            want[j, h // g] += P.T @ w
            # P's rounding; the score's 32-bit sum and the exponential (4 ulp); lse: its
            # sum of a lane's keys / 64 and of the pieces, and its own rounding; 32-bit
            # sums over the query rows
            off = u + (d + 8) * F32 * scale * float((q.abs() @ k.abs().T).max()) + 8 * F32 + \
                (k_len[b] / 64 + 64 + 4 * float(lse64.abs().max())) * F32 + \
                (g * q_len[b] / 16 + 64) * F32
            tol[j, h // g] += off * (P.T @ w.abs())
    # dV itself is rounded once (2^-25: below 2^-14)
    close(got, want.cpu(), (tol + u * want.abs() + 2.0 ** -25).cpu(), "dV")


# ---- the largest scales ------------------------------------------------------------------

@pytest.mark.parametrize("rows", ["16", "128"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [3.4e38, -3e38])
def test_largest_scales(gpu, monkeypatch, rows, dtype, scale):
    """Every finite scale is taken, also where scale log2 e is not finite in 32 bits:
    scores of 0 stay 0."""
    monkeypatch.setenv("F3S_CROSS_ROWS", rows)
    monkeypatch.setenv("F3S_PREFIX_ROWS", rows)
    gen = torch.Generator().manual_seed(2)
    u, n, kv, d = half_step(dtype), 77, 2, 64
    V = torch.randn((n, kv, d), generator=gen).to(dtype).to(DEV)
    zero = torch.zeros((3, 4, d), dtype=dtype, device=DEV)
    plan = gpu.CrossPlan([0, 3], [0, n], 4, kv, d, device=DEV)
    G = torch.ones_like(zero)
    mean = V.double().mean(0).repeat_interleave(2, 0).expand(3, 4, d).cpu()
    size = V.double().abs().mean(0).repeat_interleave(2, 0).expand(3, 4, d).cpu()
    O, lse = gpu.cross_forward(plan, zero, V, V, scale=scale)
    # (1 / n is rounded to 16 bits, in the cache to 11)
    close(O, mean, (u + 256 * F32) * size + u * mean.abs() + 2.0 ** -25, "O")
    close(lse, torch.full((3, 4), math.log(n)).double(), torch.full((3, 4), 16 * F32).double(),
          "lse")
    dV = gpu.cross_backward(plan, zero, V, V, O, G, lse, scale=scale)[2]
    want = torch.full(V.shape, 6 / n, dtype=torch.float64)
    close(dV, want, (2 * u + 256 * F32) * want, "dV")
    cache = _cache(gpu, 10, 16, kv, d)
    table, lens = torch.arange(5, 10, dtype=torch.int32, device=DEV).view(1, -1), _int32([n])
    pages = torch.arange(5, dtype=torch.int32, device=DEV)
    for t in (table, pages.view(1, -1)):
        gpu.cache_write(cache, V[None], V[None], t, lens)
    back = gpu.cache_read(cache, table, lens, n, torch.float32)[1][0].double()
    mean = back.mean(0).repeat_interleave(2, 0)[None].cpu()
    size = back.abs().mean(0).repeat_interleave(2, 0)[None].cpu()
    for k, more in ((n, {}), (2 * n, dict(prefix=pages, prefix_len=n))):
        O, lse = gpu.cache_attend(cache, zero[None, :1], table, lens, scale=scale, **more)
        close(O[0], mean, (2.0 ** -11 + 256 * F32) * size + u * mean.abs() + 2.0 ** -24 * 4, "O")
        close(lse[0], torch.full((1, 4), math.log(k)).double(),
              torch.full((1, 4), 16 * F32).double(), "lse")


# ---- small probabilities in sums ---------------------------------------------------------

@pytest.mark.parametrize("way", ["cross 16", "cross 128", "own", "prefix 16", "prefix 128"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [32, 64, 128, 160])
def test_small_probabilities(gpu, monkeypatch, way, dtype, d):
    """Every 32nd key has 2^19.64 times the probability of the others (20.5 of fp16's
    smallest steps, were it 1) and a value of zero: the result is the sum of the small
    ones, which keep their 11 bits (8 in bf16 cross attention)."""
    kind, _, rows = way.partition(" ")
    monkeypatch.setenv("F3S_CROSS_ROWS", rows or "16")
    monkeypatch.setenv("F3S_PREFIX_ROWS", rows or "16")
    gen = torch.Generator().manual_seed(d)
    u, n, kv, g = half_step(dtype), 800, 2, 2
    up = u if kind == "cross" else 2.0 ** -11
    scale = 19.64 * math.log(2)
    K, V = torch.zeros((n, kv, d)), 512 + 256 * torch.rand((n, kv, d), generator=gen)
    K[::32, :, 0], V[::32] = 1, 0
    Q = torch.zeros((3, kv * g, d))
    Q[..., 0] = 1
    Q, K, V = (x.to(dtype).to(DEV) for x in (Q, K, V))
    if kind == "cross":
        plan = gpu.CrossPlan([0, 3], [0, n], kv * g, kv, d, device=DEV)
        O, lse = gpu.cross_forward(plan, Q, K, V, scale=scale)
    else:
        page = 16
        cache = _cache(gpu, n // page + 1, page, kv, d)
        pages = torch.arange(n // page, dtype=torch.int32, device=DEV).view(1, -1)
        gpu.cache_write(cache, K[None], V[None], pages, _int32([n]))
        K, V = (x[0] for x in gpu.cache_read(cache, pages, _int32([n]), n, torch.float32))
        if kind == "own":
            table, lens, more = pages.expand(3, -1).contiguous(), [n] * 3, {}
        else:
            table, lens = torch.zeros((3, 1), dtype=torch.int32, device=DEV), [0] * 3
            more = dict(prefix=pages[0], prefix_len=n)
        O, lse = (x[:, 0] for x in gpu.cache_attend(cache, Q[:, None], table, _int32(lens),
                                                    scale=scale, **more))
    for h in range(kv * g):
        f = attention(Q[:, h].double(), K[:, h // g].double(), V[:, h // g].double(), scale, u)
        # P's rounding, the probabilities' 32-bit error, O's own rounding
        tol = (up + f["ep"][:, None]) * f["O"].abs() + u * f["O"].abs()
        close(O[:, h], f["O"].cpu(), tol.cpu(), (way, h))
        close(lse[:, h], f["lse"].cpu(), f["lse_tol"].cpu(), ("lse", way, h))


# ---- the largest scores --------------------------------------------------------------------

@pytest.mark.parametrize("way", ["cross 16", "cross 128", "own", "prefix 16", "prefix 128"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [3e4, 1e5, 1e6, 1e9, -1e5])
def test_largest_scores(gpu, monkeypatch, way, dtype, scale):
    """Scores so large that 32 bits hold no fractions of theirs, up to a key that
    outweighs all others: the result is that key's value, and the largest score the
    log-sum-exp."""
    kind, _, rows = way.partition(" ")
    monkeypatch.setenv("F3S_CROSS_ROWS", rows or "16")
    monkeypatch.setenv("F3S_PREFIX_ROWS", rows or "16")
    gen = torch.Generator().manual_seed(3)
    n, kv, g, d = 320, 1, 2, 64
    K, V = torch.zeros((n, kv, d)), torch.randn((n, kv, d), generator=gen)
    # (multiples of 64, exact in 8 bits next to each other; the largest is the last but 3)
    K[:, 0, 0] = 64.0 * (torch.arange(n) // 32 + 1)
    K[n - 3, 0, 0] = 896
    Q = torch.zeros((3, kv * g, d))
    Q[..., 0] = 1 if scale > 0 else -1
    Q, K, V = (x.to(dtype).to(DEV) for x in (Q, K, V))
    if kind == "cross":
        plan = gpu.CrossPlan([0, 3], [0, n], kv * g, kv, d, device=DEV)
        O, lse = gpu.cross_forward(plan, Q, K, V, scale=scale)
    else:
        cache = _cache(gpu, n // 16 + 1, 16, kv, d)
        pages = torch.arange(n // 16, dtype=torch.int32, device=DEV).view(1, -1)
        gpu.cache_write(cache, K[None], V[None], pages, _int32([n]))
        k, v = (x[0] for x in gpu.cache_read(cache, pages, _int32([n]), n, dtype))
        assert torch.equal(k, K)
        V = v
        if kind == "own":
            table, lens, more = pages.expand(3, -1).contiguous(), [n] * 3, {}
        else:
            table, lens = torch.zeros((3, 1), dtype=torch.int32, device=DEV), [0] * 3
            more = dict(prefix=pages[0], prefix_len=n)
        O, lse = (x[:, 0] for x in gpu.cache_attend(cache, Q[:, None], table, _int32(lens),
                                                    scale=scale, **more))
    # one weight over itself, a power of two or (128 rows) next to one: at most the
    # rounding of 16 bits, and of the quotient
    want = V[n - 3].double().expand(3, g, d).cpu()
    u = half_step(dtype)
    close(O, want, (2 * u + 4 * F32) * want.abs() + 2.0 ** -25, way)
    # the score's and the logarithm's factor, and their roundings
    close(lse, torch.full((3, g), 896 * abs(scale), dtype=torch.float64),
          torch.full((3, g), 8 * F32 * 896 * abs(scale), dtype=torch.float64), ("lse", way))
