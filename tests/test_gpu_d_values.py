"""Values of the dense operators where 16 bits of a product's operands could lose
them: tokens before one whose values are far larger."""
import math

import pytest
import torch

from _dense import attention, close, half_step
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
