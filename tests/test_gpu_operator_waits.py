"""The operators' bounded waits: with a limit of a few polls a wait runs out although everything it waits for is under way.
The call ends all the same with nothing of its own left in flight, the status word tells, and later calls give what they
gave before."""
import math

import pytest
import torch

from paper_2312_17530_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture
def polls():
    yield binding.selftest_operator_polls
    binding.selftest_operator_polls(0)


def give_up_and_recover(polls, call, outputs):
    """`call` with ever larger limits, each followed by a call without one; both have to end."""
    assert binding.operator_status() == 0
    call()
    assert binding.operator_status() == 0
    want = [t.clone() for t in outputs]
    seen = 0
    for limit in (1, 2, 3, 5, 9, 17, 33, 65, 129, 257):
        for _ in range(4):
            polls(limit)
            call()
            flags = binding.operator_status()
            assert flags in (0, binding.STATUS_TIMEOUT)
            seen |= flags
            if not flags:
                assert all(torch.equal(a, b) for a, b in zip(want, outputs))
            polls(0)
            for t in outputs:
                t.fill_(3.0)
            call()
            assert binding.operator_status() == 0
            assert all(torch.equal(a, b) for a, b in zip(want, outputs))
    return seen


def test_limits_are_checked(polls):
    for bad in (-1, (1 << 20) + 1):
        with pytest.raises(binding.RsdgcError) as e:
            polls(bad)
        assert e.value.code == binding.ERR_INVALID
    polls(1 << 20)


@pytest.mark.parametrize("n,v,d", [(60, 3000, 136), (700, 9000, 520)])
def test_head_gradient(polls, n, v, d):
    gen = torch.Generator(device="cuda").manual_seed(n)
    H = torch.randn(n, d, generator=gen, device="cuda").bfloat16()
    W = (torch.randn(v, d, generator=gen, device="cuda") * (2 / math.sqrt(d))).bfloat16()
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
    g, lse = torch.rand(n, generator=gen, device="cuda"), torch.logsumexp(H.float() @ W.float().T, 1)
    dh, dw = torch.empty_like(H), torch.empty_like(W)
    ws = torch.zeros(binding.head_workspace_bytes(n, v, d), dtype=torch.uint8, device="cuda")
    seen = give_up_and_recover(polls, lambda: binding.head_loss_backward(H, W, labels, lse, g, dh, dw, ws), (dh, dw))
    assert seen == binding.STATUS_TIMEOUT


@pytest.mark.parametrize("n,v,d,k", [(60, 3000, 136, 0), (700, 9000, 520, 0), (300, 20000, 264, 9), (60, 3000, 16384, 0),
                                     (300, 5000, 16384, 9)])
def test_head_forward(polls, n, v, d, k):
    """The warps that join a row's columns leave together, whichever of them gave up first.  (A poll waits some microseconds
    by itself: short contractions are over before the first ends.)"""
    gen = torch.Generator(device="cuda").manual_seed(n)
    H = torch.randn(n, d, generator=gen, device="cuda").bfloat16()
    W = (torch.randn(v, d, generator=gen, device="cuda") * (2 / math.sqrt(d))).bfloat16()
    ws = torch.zeros(binding.head_workspace_bytes(n, v, d, max(k, 1)), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    if k:
        index = torch.randint(0, v, (n, k), generator=gen, device="cuda")
        logit = torch.randn(n, k, generator=gen, device="cuda")
        call = lambda: binding.head_distill_forward(H, W, index, logit, 2.0, loss, lse, ws)  # noqa: E731
    else:
        labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
        call = lambda: binding.head_loss_forward(H, W, labels, loss, lse, ws)  # noqa: E731
    seen = give_up_and_recover(polls, call, (loss, lse))
    assert seen == binding.STATUS_TIMEOUT or d < 16384


@pytest.mark.parametrize("kind,n,d", [(torch.float32, 2000, 1000), (torch.float32, 3000, 8200), (torch.bfloat16, 6000, 4100),
                                      (torch.bfloat16, 6000, 8192), (torch.float16, 3000, 16500)])
def test_layer_norm(polls, kind, n, d):
    """Rows through the rings, the teams' and the clusters'."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, dy = (torch.randn(n, d, generator=gen, device="cuda").to(kind) for _ in range(2))
    w = torch.randn(d, generator=gen, device="cuda").to(kind)
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    give_up_and_recover(polls, lambda: binding.layer_norm_forward(x, w, None, y, mean, rstd), (y, mean, rstd))
    binding.layer_norm_forward(x, w, None, y, mean, rstd)
    ws = torch.zeros(binding.layer_norm_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
    give_up_and_recover(polls, lambda: binding.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, ws), (dx, dw, db))


def test_status_is_reported_once_and_by_any_stream():
    assert binding.operator_status() == 0
    binding.selftest_operator_wait(300)
    assert binding.operator_status() == binding.STATUS_TIMEOUT and binding.operator_status() == 0
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        binding.selftest_operator_wait(10)
    side.synchronize()
    assert binding.operator_status() == binding.STATUS_TIMEOUT and binding.operator_status() == 0
    for bad in (0, -1, (1 << 20) + 1):
        with pytest.raises(binding.RsdgcError) as e:
            binding.selftest_operator_wait(bad)
        assert e.value.code == binding.ERR_INVALID


def test_no_status_is_lost_between_reading_and_clearing():
    """Waits run out on one stream while another asks all the time: each of them is reported at the latest when all is over, and a
    report that found nothing clears nothing."""
    side, asks = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(50):
        with torch.cuda.stream(side):
            binding.selftest_operator_wait(1)
        told = 0
        with torch.cuda.stream(asks):
            while not side.query():
                told |= binding.operator_status()
            told |= binding.operator_status()
        assert told == binding.STATUS_TIMEOUT
    assert binding.operator_status() == 0
