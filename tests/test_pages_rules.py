"""Which calls of the page tables one workgroup does by itself: those need no workspace."""
import pytest

from paper_2505_08098_amd import dense


@pytest.mark.parametrize("B,pages,n,alone", [
    (256, 126, 5, True), (1024, 128, 32, True), (8, 500, 256, True), (1, 500, 2048, True),
    (31, 500, 64, True), (64, 500, 32, True),
    # a prompt's part for each of many sequences: 43 us instead of 12
    (64, 500, 64, False), (64, 500, 256, False), (256, 126, 64, False), (62, 500, 33, True),
    (63, 500, 33, False), (1, 500, 2049, False),
])
def test_alone(B, pages, n, alone):
    size = dense._lib().f3s_pages_assign_workspace_bytes(B, pages, n)
    assert (size == 0) == alone
