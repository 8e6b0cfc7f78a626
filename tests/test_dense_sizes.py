"""Sizes beyond 32 bits through the binding: refused, not taken modulo 2^32."""
import pytest
import torch

from paper_2505_08098_amd import dense


@pytest.mark.parametrize("kw", [
    dict(heads=2**32 + 4), dict(kv_heads=2**32 + 2), dict(d=2**32 + 64), dict(heads=2**31),
    dict(heads=-(2**32) + 4),
])
def test_plan_sizes(kw):
    with pytest.raises(ValueError):
        dense.CrossPlan([0, 2], [0, 3], **{"heads": 4, "kv_heads": 2, "d": 64, **kw})


@pytest.mark.gpu
def test_prefix_beyond_32_bits(gpu):
    """A prefix of 2^32 + 5 tokens, whose pages are there, is not one of 5."""
    dev = torch.device("cuda:0")
    cache = gpu.Cache.empty(2, 256, 1, 32)
    prefix = torch.zeros((1 << 24) + 1, dtype=torch.int32, device=dev)
    table, lens = torch.ones((1, 1), dtype=torch.int32, device=dev), prefix[:1]
    Q = torch.zeros((1, 1, 1, 32), dtype=torch.float16, device=dev)
    for n in (2**32 + 5, 2**32, 2**31):
        with pytest.raises(ValueError):
            gpu.cache_attend(cache, Q, table, lens, prefix=prefix, prefix_len=n)
    with pytest.raises(gpu.F3SError):           # (beyond 2^30, which 32 bits hold)
        gpu.cache_attend(cache, Q, table, lens, prefix=prefix, prefix_len=2**30 + 1)


@pytest.mark.gpu
def test_read_beyond_32_bits(gpu):
    dev = torch.device("cuda:0")
    cache = gpu.Cache.empty(2, 16, 1, 32)
    table, lens = (torch.zeros(s, dtype=torch.int32, device=dev) for s in ((0, 1), (0,)))
    with pytest.raises(ValueError):
        gpu.cache_read(cache, table, lens, 2**32 + 1)
