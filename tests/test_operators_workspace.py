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


@pytest.mark.parametrize("v", [1, 500, 2048, 2049, 20000, 128000, 600000])
@pytest.mark.parametrize("d", [8, 512, 513, 2000, 8192, 20000])
def test_head_workspace_does_for_fewer_tokens(v, d):
    """The last batch is often a smaller one."""
    size = binding.lib().rsdgc_head_workspace_bytes
    n = list(range(0, 1600)) + list(range(1600, 40000, 509)) + [16383, 16384, 16385, 32768, 32769]
    got = [size(t, v, d, 3) for t in sorted(n)]
    assert got[0] >= 0 and got == sorted(got)
    for t in (1, 100, 128, 129, 2000):
        assert size(t, v, d, 1) <= size(t, v, d, 2) <= size(t, v, d, 100)


def test_head_workspace_stays_small():
    size = binding.head_workspace_bytes
    assert size(64, 8000, 512) <= 16 << 20            # two planes of dz, dhidden's parts
    assert size(2048, 32000, 2048) <= 300 << 20       # two pieces of dz, dhidden's parts
    assert size(8192, 128000, 4096) <= 500 << 20


def test_example_says_what_it_does_not_take():
    from paper_2312_17530_b200 import lm_step

    for bad in (dict(width=100), dict(width=0), dict(n_tokens=1), dict(n_top=0), dict(vocab=10, n_top=11), dict(n_top=1025)):
        with pytest.raises(ValueError):
            lm_step.run(**bad)


def test_scoring_needs_what_the_forward_pass_uses():
    """A pair of binary32 per token and 128 entries of the vocabulary, the targets, and little more."""
    size, train = binding.head_forward_workspace_bytes, binding.head_workspace_bytes
    for n, v, d, k in ((1, 1, 1, 1), (64, 8000, 512, 8), (8192, 128000, 4096, 1), (333, 10007, 776, 1024)):
        least = 8 * n * -(-v // 128) + 12 * n * k
        assert least <= size(n, v, d, k) <= least + 4 * n + 4 * -(-v // 2048) + 4096
        assert size(n, v, d, k) <= train(n, v, d, k) and size(n, v, d, k) <= size(n + 1, v, d, k)
    for bad in ((-1, 10, 10, 1), (1, 0, 10, 1), (1, 10, 10, 0), (1, 10, 10, 1025)):
        with pytest.raises(binding.RsdgcError):
            size(*bad)
