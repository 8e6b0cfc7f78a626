"""Registers of the dense operators' kernels, from the metadata of the built code
objects: no instance spills, and each leaves room for the waves per SIMD that its
launch bounds and the division of the work count with."""
import re

import pytest

from test_kernel_resources import _room, kernels  # noqa: F401  (a fixture)

HEADS = (32, 64, 96, 128, 160, 192, 224, 256)
THREE = {d: 3 if d <= 64 else 2 if d <= 128 else 1 for d in HEADS}
ROOM = {
    "k_cross_many": THREE,
    "k_attend_prefix": THREE,
    "k_cross_dkv": THREE,
    "k_cross_dq": {**THREE, 32: 4},
    "k_cross_few": {**THREE, 32: 4},
    "k_attend": {d: 4 if d <= 64 else 3 if d <= 160 else 2 for d in HEADS},
}


@pytest.mark.parametrize("kernel", sorted(ROOM))
def test_attention_kernels(kernels, kernel):  # noqa: F811
    seen = set()
    for name, (registers, spilled) in kernels.items():
        m = re.search(r"\d%sILi(\d+)ELi(\d)EE" % kernel, name)
        if not m:
            continue
        d, dtype = (int(x) for x in m.groups())
        assert spilled == 0, (name, spilled)
        assert _room(registers) >= ROOM[kernel][d], (name, registers)
        seen.add((d, dtype))
    assert len(seen) == 2 * len(HEADS)


@pytest.mark.parametrize("kernel,instances", [("k_cross_join", 32), ("k_attend_join", 32),
                                              ("k_cross_sum", 32), ("k_cache_write", 16),
                                              ("k_cache_read", 24)])
def test_kernels_that_stream(kernels, kernel, instances):  # noqa: F811
    """Joins and the cache's rows: bound by bytes in flight, so four waves at least."""
    found = [v for name, v in kernels.items() if re.search(r"\d%sI" % kernel, name)]
    assert len(found) == instances
    assert all(spilled == 0 and _room(registers) >= 4 for registers, spilled in found)
