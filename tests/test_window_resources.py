"""Registers of the window and masked-cache kernels, from the metadata of the built code
objects: no instance spills, and each leaves room for the waves per SIMD that its launch
bounds and the division of the work count with."""
import re

import pytest

from test_dense_resources import HEADS, THREE
from test_kernel_resources import _room, kernels  # noqa: F401  (a fixture)

FEW = {d: 4 if d <= 64 else 3 if d <= 160 else 2 for d in HEADS}
ROOM = {
    "k_attend_window": FEW,
    "k_attend_tree": FEW,
    "k_attend_own14": THREE,     # a window's and a tree's instances, four and eight waves
    "k_attend_own24": THREE,
    "k_attend_own18": {96: 2, 128: 2},
    "k_attend_own28": {96: 2, 128: 2},
    "k_window": THREE,
    "k_window_dq": {**THREE, 32: 4},
    "k_window_dkv": THREE,
}


@pytest.mark.parametrize("kernel", sorted(ROOM))
def test_attention_kernels(kernels, kernel):  # noqa: F811
    seen, wrong = set(), []
    for name, (registers, spilled) in kernels.items():
        of, mask = kernel, ""
        if kernel[-1].isdigit():
            of, mask = kernel[:-2], "Li%sELi%sE" % (kernel[-2], kernel[-1])
        m = re.search(r"\d%sILi(\d+)ELi(\d)E%sE" % (of, mask), name)
        if not m:
            continue
        d, dtype = (int(x) for x in m.groups())
        if spilled or _room(registers) < ROOM[kernel][d]:
            wrong.append((d, dtype, registers, spilled))
        seen.add((d, dtype))
    assert not wrong
    assert len(seen) == 2 * len(ROOM[kernel])
