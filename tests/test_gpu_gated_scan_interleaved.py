"""Results that lie between one another without overlapping, other than sequences or steps first."""
import pytest
import torch

from paper_2312_17530_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,t,seq,step", [(2, 2, 192, 128), (3, 4, 64, 192), (5, 3, 128, 704), (2, 7, 192, 128), (2, 8, 160, 128)])
def test_rows_between_one_another(n, t, seq, step):
    """A step of 128 and a sequence of 192 apart: rows at 0, 128, 192, 320, and with seven steps one gap filled after the other.  The last size overlaps and is refused."""
    d = 64
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, gate = (torch.randn(n, t, d, generator=gen, device="cuda") for _ in range(2))
    want = torch.empty_like(x)
    binding.gated_scan_forward(x, gate, want)
    buf = torch.full(((n - 1) * seq + (t - 1) * step + d,), 7.0, device="cuda")
    y = torch.as_strided(buf, (n, t, d), (seq, step, 1))
    if (n, t) == (2, 8):
        with pytest.raises(binding.RsdgcError):
            binding.gated_scan_forward(x, gate, y)
        assert (buf == 7.0).all()
        return
    binding.gated_scan_forward(x, gate, y)
    assert torch.equal(y, want)
    y.fill_(7.0)
    assert (buf == 7.0).all() and binding.operator_status() == 0
