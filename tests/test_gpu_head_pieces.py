"""The head's gradient over three pieces of the vocabulary: the third writes again into the first one's dz buffer, is the
second to be added to dhidden, and its launch takes its tiles from the third queue.  How many pieces a call had follows from
the kernels that it launched."""
import math

import pytest
import torch

from paper_2312_17530_b200 import binding
from test_gpu_head import TYPES, label_want, operand, output, top_want, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,d,k", [(33000, 5000, 24, 0), (20000, 9000, 40, 7)])
def test_three_pieces(kind, n, v, d, k):
    gen = torch.Generator(device="cuda").manual_seed(n)
    dtype = TYPES[kind]
    H, W = operand(gen, n, d, dtype), operand(gen, v, d, dtype, 0, 2 / math.sqrt(d))
    g = torch.rand(n, generator=gen, device="cuda") / n * (1024 if kind == "f16" else 1)
    dh, dw = output(n, d, dtype, d), output(v, d, dtype, d)
    loss, lse, ws = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), workspace(n, v, d, max(k, 1))
    if k:
        index = torch.randint(0, v, (n, k), generator=gen, device="cuda")
        logit = torch.randn(n, k, generator=gen, device="cuda")
        binding.head_distill_forward(H, W, index, logit, 2.0, loss, lse, ws)
        want = top_want(H, W, index, logit, 2.0)
    else:
        labels = torch.randint(-1, v, (n,), generator=gen, device="cuda")
        binding.head_loss_forward(H, W, labels, loss, lse, ws)
        want = label_want(H, W, labels)
    ws.fill_(0xFF)
    before = binding.launch_count()
    if k:
        binding.head_distill_backward(H, W, index, logit, 2.0, lse, g, dh, dw, ws)
    else:
        binding.head_loss_backward(H, W, labels, lse, g, dh, dw, ws)
    # the targets, the scale, a launch per piece and one more, dhidden's sum in grids of 32768 rows at most
    pieces = binding.launch_count() - before - (1 if k else 0) - 1 - 1 - -(-n // 32768)
    assert pieces == 3
    assert binding.operator_status() == 0
    want.check_forward(loss, lse)
    want.check_backward(g, dh, dw, dtype, pieces)
    # the same bits once more, from a workspace that holds the last call's
    first = dh.clone(), dw.clone()
    if k:
        binding.head_distill_backward(H, W, index, logit, 2.0, lse, g, dh, dw, ws)
    else:
        binding.head_loss_backward(H, W, labels, lse, g, dh, dw, ws)
    assert torch.equal(first[0], dh) and torch.equal(first[1], dw)


@pytest.mark.parametrize("k", [0, 11])
def test_scoring_stays_inside_its_workspace(k):
    n, v, d = 3000, 9001, 72
    gen = torch.Generator(device="cuda").manual_seed(3)
    H, W = operand(gen, n, d, torch.bfloat16), operand(gen, v, d, torch.bfloat16, 0, 0.2)
    size = binding.head_forward_workspace_bytes(n, v, d, max(k, 1))
    assert size < binding.head_workspace_bytes(n, v, d, max(k, 1)) // 4
    space = torch.full((size + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    if k:
        index = torch.randint(0, v, (n, k), generator=gen, device="cuda")
        logit = torch.randn(n, k, generator=gen, device="cuda")
        call = lambda ws: binding.head_distill_forward(H, W, index, logit, 2.0, loss, lse, ws)  # noqa: E731
        want = top_want(H, W, index, logit, 2.0)
    else:
        labels = torch.randint(-1, v, (n,), generator=gen, device="cuda")
        call = lambda ws: binding.head_loss_forward(H, W, labels, loss, lse, ws)  # noqa: E731
        want = label_want(H, W, labels)
    call(space[:size])
    want.check_forward(loss, lse)
    assert (space[size:] == 0xFF).all() and binding.operator_status() == 0
    with pytest.raises(ValueError):
        call(space[:size - 1])
    with pytest.raises(ValueError):  # the gradient needs more
        binding.head_loss_backward(H, W, torch.zeros(n, dtype=torch.int64, device="cuda"), lse, loss, H.clone(), W.clone(),
                                   space[:size])
