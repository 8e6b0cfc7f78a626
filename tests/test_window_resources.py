"""Registers of the window and masked-cache kernels, from the metadata of the built code
objects: no instance spills, and each leaves room for the waves per SIMD that its launch
bounds and the division of the work count with."""
import re

import pytest

from test_dense_resources import HEADS, THREE
from test_kernel_resources import _room, kernels  # noqa: F401  (a fixture)

ROOM = {
    "k_window": THREE,
    "k_window_dq": {**THREE, 32: 4},
    "k_window_dkv": THREE,
}


@pytest.mark.parametrize("kernel", sorted(ROOM))
def test_attention_kernels(kernels, kernel):  # noqa: F811
    seen, wrong = set(), []
    for name, (registers, spilled) in kernels.items():
        m = re.search(r"\d%sILi(\d+)ELi(\d)EE" % kernel, name)
        if not m:
            continue
        d, dtype = (int(x) for x in m.groups())
        if spilled or _room(registers) < ROOM[kernel][d]:
            wrong.append((d, dtype, registers, spilled))
        seen.add((d, dtype))
    assert not wrong
    assert len(seen) == 2 * len(HEADS)
