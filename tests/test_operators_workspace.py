"""What the layer norm's gradient asks of its caller: room for the partial sums that it can write, no more."""
import pytest

from paper_2312_17530_b200 import binding
from paper_2312_17530_b200.build import build_library


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


def test_layer_norm_workspace_follows_the_rows():
    """Two binary32 sums per column and slot.  A row takes one slot and slots come in eights; 148 for rows wider than a warp's, 3 x
    148 for a warp's rows, eight to a slot."""
    size = binding.layer_norm_workspace_bytes
    slot = 2 * 4 * 8192
    assert size(1, 8192) == 8 * slot and size(9, 8192) == 16 * slot
    assert size(148, 8192) == size(1184, 8192) == 152 * slot
    assert size(3000, 8192) == 376 * slot
    assert size(3552, 8192) == size(1 << 30, 8192) == 448 * slot
    assert size(4, 1 << 20) <= 64 << 20
    rows = [1, 2, 7, 8, 9, 63, 100, 148, 149, 1000, 1184, 1185, 3000, 3551, 4000, 1 << 20]
    assert sorted(size(n, 100) for n in rows) == [size(n, 100) for n in rows]
