"""The orthogonalised update's bounded waits, and two updates at once: see test_gpu_operator_waits.py."""
import pytest
import torch

from paper_2312_17530_b200 import binding
from test_gpu_operator_waits import give_up_and_recover

pytestmark = pytest.mark.gpu


@pytest.fixture
def polls():
    yield binding.selftest_operator_polls
    binding.selftest_operator_polls(0)


@pytest.mark.parametrize("n,m,k,out", [(1, 60, 3000, torch.bfloat16), (3, 300, 400, torch.float16), (1, 1100, 1500, torch.bfloat16),
                                       (1, 5000, 300, torch.bfloat16)])
def test_a_wait_that_gives_up(polls, n, m, k, out):
    """(Whether one does depends on how long a poll takes: the calls have to end and later ones to be right either way.)"""
    x = torch.randn(n, m, k, generator=torch.Generator(device="cuda").manual_seed(m), device="cuda")
    result = torch.empty(n, m, k, dtype=out, device="cuda")
    ws = torch.empty(binding.orthogonalize_workspace_bytes(n, m, k, out), dtype=torch.uint8, device="cuda")
    give_up_and_recover(polls, lambda: binding.orthogonalize(x, result, ws), (result,))


def test_two_at_once():
    """On two streams, each with its workspace, of sizes that take different numbers of multiprocessors."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    calls = []
    for m, k in ((700, 900), (64, 64), (2000, 300)):
        x = torch.randn(m, k, generator=gen, device="cuda")
        out = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(binding.orthogonalize_workspace_bytes(1, m, k, torch.bfloat16), dtype=torch.uint8, device="cuda")
        binding.orthogonalize(x, out, ws)
        calls.append((x, out, ws, out.clone(), torch.cuda.Stream()))
    for c in calls:
        c[1].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for x, out, ws, _, stream in calls:
            with torch.cuda.stream(stream):
                binding.orthogonalize(x, out, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(c[1], c[3]) for c in calls)
    assert binding.operator_status() == 0


@pytest.mark.parametrize("m,k", [(100, 300), (600, 500)])
def test_rows_and_matrices_with_gaps(m, k):
    """A stack of every second matrix of a wider arena, into every second row's start; what lies between stays."""
    gen = torch.Generator(device="cuda").manual_seed(m)
    big = torch.randn(6, m, k + 11, generator=gen, device="cuda")
    x = big[::2, :, 3:3 + k]
    place = torch.full((3, 2 * m, k + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    out = place[:, ::2, 1:1 + k]
    ws = torch.empty(binding.orthogonalize_workspace_bytes(3, m, k, torch.bfloat16), dtype=torch.uint8, device="cuda")
    binding.orthogonalize(x, out, ws)
    plain = torch.empty(3, m, k, dtype=torch.bfloat16, device="cuda")
    binding.orthogonalize(x.contiguous(), plain, ws)
    assert torch.equal(out, plain) and binding.operator_status() == 0
    out.fill_(7.0)
    assert (place == 7.0).all()
