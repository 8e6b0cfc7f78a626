"""The 8-bit cache on the GPU: writing and reading back against the format's
definition, bit by bit; attention over the cache against plain 64-bit
attention."""
import math

import pytest
import torch

from _dense import attention, close, code_values, half_step, quantised, two_to

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
TYPES = [torch.float16, torch.bfloat16]


def _table(gen, B, pages, first=0, spare=3):
    """[B, pages] of distinct pages in no order, and the number of pages."""
    n = first + B * pages + spare
    order = first + torch.randperm(n - first, generator=gen)[: B * pages]
    return order.to(torch.int32).view(B, pages), n


def _cache(gpu, n_pages, page, kv, d, fill=0x7F):
    """Pages that hold ``fill`` (NaN codes) and large powers where nothing is
    written."""
    shape = (n_pages, kv, page, d)
    codes = [torch.full(shape, fill, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
             for _ in range(2)]
    powers = [torch.full(shape[:3], 250, dtype=torch.uint8, device=DEV) for _ in range(2)]
    return gpu.Cache(*codes, *powers)


def _rows(gen, shape, dtype):
    x = torch.randn(shape, generator=gen, dtype=torch.float64)
    return (x * torch.exp(torch.randn(shape[-1], generator=gen, dtype=torch.float64))).to(dtype)


def _values(cache):
    """(K, V) of every place of the cache in 64 bits, on the host."""
    code = code_values()
    out = []
    for c, e in ((cache.k, cache.k_exp), (cache.v, cache.v_exp)):
        v = code[c.view(torch.uint8).cpu().long()]
        out.append(v * two_to(e.cpu().long() - 127)[..., None])
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,page,kv,lens,n", [
    (64, 16, 2, [1, 5, 16, 17, 40], 1),
    (32, 32, 1, [33, 7, 64], 33),
    (128, 64, 3, [100, 65, 300, 1], 65),
    (96, 16, 2, [50, 16], 20),
    (256, 128, 1, [129, 128], 2),
    (160, 16, 1, [3], 3), (192, 256, 2, [300], 7), (224, 32, 1, [31], 31),
])
def test_write_and_read(gpu, dtype, d, page, kv, lens, n):
    gen = torch.Generator().manual_seed(d + page + n)
    B = len(lens)
    table, n_pages = _table(gen, B, -(-max(lens) // page))
    K, V = _rows(gen, (B, n, kv, d), dtype), _rows(gen, (B, n, kv, d), dtype)
    K[0, -1, 0] = 0                      # a row of zeros
    V[-1, -1, 0] *= 2.0 ** -12           # small ones
    V[0, -1, 0, :2] = torch.tensor([math.nan, -math.inf])
    cache = _cache(gpu, n_pages, page, kv, d)
    before = _values(cache)
    gpu.cache_write(cache, K.to(DEV), V.to(DEV), table.to(DEV),
                    torch.tensor(lens, dtype=torch.int32, device=DEV))
    after = _values(cache)
    powers = [cache.k_exp.cpu(), cache.v_exp.cpu()]
    back = gpu.cache_read(cache, table.to(DEV), torch.tensor(lens, dtype=torch.int32).to(DEV),
                          n, dtype)
    back32 = gpu.cache_read(cache, table.to(DEV),
                            torch.tensor(lens, dtype=torch.int32).to(DEV), n, torch.float32)
    for x, old, new, power, got, got32 in zip((K, V), before, after, powers, back, back32):
        want, e = quantised(x)
        there = torch.zeros(old.shape[:3], dtype=torch.bool)
        for b, m in enumerate(lens):
            for t in range(n):
                p = m - n + t
                if p < 0:
                    assert not got[b, t].any() and not got32[b, t].any()
                    continue
                at = int(table[b, p // page]), slice(None), p % page
                there[at] = True
                assert torch.equal(new[at].nan_to_num(9e9), want[b, t].nan_to_num(9e9))
                assert torch.equal(power[at], e[b, t])
                assert torch.equal(got[b, t].cpu().nan_to_num(9), want[b, t].to(dtype)
                                   .nan_to_num(9))
                assert torch.equal(got32[b, t].double().cpu().nan_to_num(9),
                                   want[b, t].nan_to_num(9))
        # every other place is as it was
        assert torch.equal(new[~there].nan_to_num(9e9), old[~there].nan_to_num(9e9))
        assert bool((power[~there] == 250).all())


def test_every_16_bit_value(gpu):
    """All finite values of both types, a row each of one value and its
    neighbours: the power and the codes at every border."""
    for dtype in TYPES:
        bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
        x = bits.view(dtype)
        x = x[torch.isfinite(x)]
        x = x[: len(x) // 32 * 32].view(1, -1, 1, 32)
        # columns of other magnitudes in the same row
        y = torch.cat([x, x.flip(1)], -1).contiguous()
        n = y.shape[1]
        pages = -(-n // 256)
        cache = _cache(gpu, pages, 256, 1, 64)
        table = torch.arange(pages, dtype=torch.int32, device=DEV).view(1, -1)
        lens = torch.tensor([n], dtype=torch.int32, device=DEV)
        gpu.cache_write(cache, y.to(DEV), y.flip(-1).contiguous().to(DEV), table, lens)
        K, V = gpu.cache_read(cache, table, lens, n, torch.float32)
        want, e = quantised(y)
        # (the largest bfloat16 values are nearest to code 256 of power 120:
        # 2^128, which 32 bits hold as infinity)
        want = want.float()
        assert torch.equal(K.cpu(), want)
        assert torch.equal(V.cpu(), want.flip(-1))
        got = cache.k_exp.cpu().view(-1)[:n]
        assert torch.equal(got, e.view(-1))


def _attend_case(gpu, dtype, d, page, kv, g, lens, n, prefix_len, scale=None, seed=0, room=0):
    gen = torch.Generator().manual_seed(seed + d + page + n)
    B = len(lens)
    shared = -(-prefix_len // page)
    table, n_pages = _table(gen, B, max(1, -(-max(max(lens), room) // page)), first=shared)
    cache = _cache(gpu, n_pages, page, kv, d)
    lens_d = torch.tensor(lens, dtype=torch.int32, device=DEV)
    prefix = None
    if prefix_len:
        prefix = torch.arange(shared - 1, -1, -1, dtype=torch.int32, device=DEV)
        x = [_rows(gen, (1, prefix_len, kv, d), dtype).to(DEV) for _ in "KV"]
        gpu.cache_write(cache, *x, prefix.view(1, -1),
                        torch.tensor([prefix_len], dtype=torch.int32, device=DEV))
    if max(lens):
        x = [_rows(gen, (B, max(lens), kv, d), dtype).to(DEV) for _ in "KV"]
        gpu.cache_write(cache, *x, table.to(DEV), lens_d)
    Q = torch.randn((B, n, kv * g, d), generator=gen, dtype=torch.float64).to(dtype)
    scale = 1 / math.sqrt(d) if scale is None else scale
    O, lse = gpu.cache_attend(cache, Q.to(DEV), table.to(DEV), lens_d, prefix=prefix,
                              prefix_len=prefix_len, scale=scale)
    torch.cuda.synchronize()
    _compare(cache, Q, table, lens, prefix, prefix_len, scale, O, lse)
    return cache, Q, table, lens_d, prefix, O, lse


def _compare(cache, Q, table, lens, prefix, prefix_len, scale, O, lse):
    dtype, page = Q.dtype, cache.page_size
    B, n, H, d = Q.shape
    g = H // cache.kv_heads
    values = _values(cache)

    def rows(pages, m):
        at = torch.arange(m)
        ok = (pages >= 0) & (pages < cache.n_pages)
        k = pages[at // page].long()
        there = ok[at // page]
        return [torch.where(there[:, None, None], x[k.clamp(0, cache.n_pages - 1), :, at % page],
                            0.0) for x in values] + [there]

    front = rows(prefix.cpu(), prefix_len) if prefix_len else None
    cap = table.shape[1] * page
    for b in range(B):
        m = min(max(lens[b], 0), cap)
        k, v, there = rows(table[b], m)
        at = torch.arange(m) + prefix_len
        if front:
            k, v, there = (torch.cat([x, y]) for x, y in zip(front, (k, v, there)))
            at = torch.cat([torch.full((prefix_len,), -1), at])
        last = prefix_len + max(lens[b], 0) - n + torch.arange(n)
        seen = (at <= last[:, None]) & there
        # a probability below the smallest f16 next to the largest power
        top = v.abs().amax((0, 2)) if len(v) else torch.zeros(cache.kv_heads)
        for h in range(H):
            # (relative to the largest value's power, of at most 2^-8 of it)
            size = 2.0 ** -25 * torch.ones(len(v), 1) * float(top[h // g]) * 2 / 448
            f = attention(Q[b, :, h].double(), k[:, h // g], v[:, h // g], scale,
                          half_step(dtype), up=2.0 ** -11, seen=seen,
                          floor=size * 448)
            what = (b, h, lens[b])
            close(O[b, :, h], f["O"], f["O_tol"], ("O",) + what)
            close(lse[b, :, h], f["lse"], f["lse_tol"], ("lse",) + what)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,page,kv,g,lens,n,prefix", [
    (64, 16, 2, 1, [1, 0, 5, 33, 16, 17], 1, 0),
    (64, 16, 1, 4, [300, 1, 64, 65], 1, 0),
    (128, 64, 2, 4, [1000, 3, 517], 1, 0),
    (128, 32, 2, 4, [100, 0, 31, 700], 1, 77),
    (32, 16, 3, 1, [40, 41], 5, 0),
    (64, 32, 1, 5, [40, 3, 0], 7, 33),      # tokens before the start see the prefix only
    (96, 16, 1, 2, [90], 3, 16),
    (256, 256, 1, 3, [600, 20], 2, 300),
    (160, 128, 1, 1, [129], 1, 1), (192, 64, 1, 2, [64], 4, 65), (224, 16, 1, 1, [15], 1, 15),
    (64, 16, 1, 40, [70, 200], 1, 50),      # rows of a sequence in several blocks
    (64, 16, 1, 3, [0, 0], 2, 0),           # no key at all
])
def test_attend(gpu, dtype, d, page, kv, g, lens, n, prefix):
    _attend_case(gpu, dtype, d, page, kv, g, lens, n, prefix)


@pytest.mark.parametrize("d,page,kv,g,lens,n", [
    (64, 16, 2, 1, [1, 0, 5, 33, 16, 17], 1), (64, 16, 1, 4, [300, 1, 64, 65], 1),
    (128, 64, 2, 4, [1000, 3, 517], 1), (32, 16, 3, 1, [40, 41], 5),
    (96, 16, 1, 2, [290], 3), (256, 256, 1, 3, [600, 20], 2),
    (64, 16, 1, 40, [570, 200], 1), (64, 16, 1, 3, [0, 0], 2), (160, 128, 1, 1, [1500], 9),
    (64, 32, 2, 8, [4000, 70, 1], 2)])
@pytest.mark.parametrize("dtype", TYPES)
def test_attend_in_pieces(gpu, dtype, d, page, kv, g, lens, n):
    """Tables with room for more than one workgroup walks: pieces, whatever the
    lengths are, and none of it where there is room for 896 keys."""
    _attend_case(gpu, dtype, d, page, kv, g, lens, n, 0, room=3000)
    short = [min(m, 896) for m in lens]
    _attend_case(gpu, dtype, d, page, kv, g, short, n, 0, room=896)


@pytest.mark.parametrize("rows", ["16", "128"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,page,kv,g,B,n,prefix", [
    (64, 16, 2, 4, 20, 1, 130),            # 80 rows
    (128, 64, 1, 8, 33, 1, 1000),          # 264 rows, a tile that is not full
    (128, 32, 2, 4, 5, 5, 321),
    (96, 16, 1, 5, 14, 1, 64), (32, 32, 1, 1, 129, 1, 63),
    (256, 128, 1, 2, 40, 1, 300), (160, 16, 1, 3, 30, 1, 65),
    (64, 16, 1, 1, 70, 1, 4500),           # more keys than one workgroup walks
])
def test_attend_shared_prefix(gpu, monkeypatch, rows, dtype, d, page, kv, g, B, n, prefix):
    """The prefix by the kernel of 16 query rows and by that of 128."""
    monkeypatch.setenv("F3S_PREFIX_ROWS", rows)
    lens = [(7 * b) % 50 for b in range(B)]
    _attend_case(gpu, dtype, d, page, kv, g, lens, n, prefix)
