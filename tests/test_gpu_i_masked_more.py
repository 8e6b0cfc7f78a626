"""More of attention over the 8-bit cache with a window or a tree of drafted tokens, on the GPU
against plain 64-bit attention: trees that end inside a tile of keys."""
import pytest
import torch

from test_gpu_g_masked import _tree_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [225, 256])
@pytest.mark.parametrize("rows", ["16", "128"])
def test_trees_that_end_inside_a_tile(gpu, monkeypatch, rows, n, d):
    """The last tile's second half lies behind the last token that a tree can have."""
    monkeypatch.setenv("F3S_OWN_ROWS", rows)
    _tree_case(gpu, torch.float16, d, 16, 1, 1, [257, 288, 321, 10, 230], n, 0, "random")
    _tree_case(gpu, torch.float16, d, 16, 1, 1, [257, 288, 321, 10, 230], n, 33, "random")
