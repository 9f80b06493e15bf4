"""Operands of more than 2^31 values: the last rows give the bits that they give in a small call of their own."""
import pytest
import torch

from paper_2312_17530_b200 import binding

pytestmark = pytest.mark.gpu


def fill(t, seed):
    """Normal values, a part at a time."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for part in t.split(1 << 15):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    return t


@pytest.mark.parametrize("d", [8192, 8193])
def test_layer_norm(d):
    n, last = 270000, 1000
    assert n * d > 1 << 31
    x, dy = (fill(torch.empty(n, d, dtype=torch.bfloat16, device="cuda"), s) for s in (1, 2))
    w = torch.randn(d, device="cuda").bfloat16()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    binding.layer_norm_forward(x, w, None, y, mean, rstd)
    binding.layer_norm_backward(dy, x, w, mean, rstd, dx)
    rows = slice(n - last, n)
    y2, dx2 = torch.empty_like(y[rows]), torch.empty_like(y[rows])
    mean2, rstd2 = torch.empty(last, device="cuda"), torch.empty(last, device="cuda")
    binding.layer_norm_forward(x[rows], w, None, y2, mean2, rstd2)
    binding.layer_norm_backward(dy[rows], x[rows], w, mean2, rstd2, dx2)
    assert torch.equal(y[rows], y2) and torch.equal(mean[rows], mean2) and torch.equal(rstd[rows], rstd2)
    assert torch.equal(dx[rows], dx2)
    assert binding.operator_status() == 0


@pytest.mark.parametrize("pitch", [4096, 4097])
def test_head(pitch):
    """A vocabulary matrix and its gradient beyond 2^31 values; labels among the last entries, whose rows of dweight follow from
    the formula: with equal logits everywhere but at the labels, dz is known."""
    n, v, d = 70, 560000, 4096
    assert v * d > 1 << 31
    W = torch.zeros(v, d, dtype=torch.bfloat16, device="cuda")
    H = torch.randn(n, d, device="cuda").bfloat16()
    labels = v - 1 - torch.arange(n, device="cuda")
    W[labels, torch.arange(n, device="cuda")] = 1.0
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    g = torch.ones(n, device="cuda")
    ws = torch.empty(binding.head_workspace_bytes(n, v, d), dtype=torch.uint8, device="cuda")
    dh = torch.empty_like(H)
    dw = torch.full((v * pitch,), 7.0, dtype=torch.bfloat16, device="cuda").view(v, pitch)
    binding.head_loss_forward(H, W, labels, loss, lse, ws)
    binding.head_loss_backward(H, W, labels, lse, g, dh, dw[:, :d], ws)
    assert binding.operator_status() == 0
    tail = v - n
    z = H.double() @ W[tail:].double().T                    # all other logits are zero
    want = torch.logsumexp(torch.cat([z, torch.full((n, 1), float(torch.tensor(float(tail)).log()), device="cuda")], 1), 1)
    assert ((lse.double() - want).abs() <= 2.0 ** -18 * want.abs()).all()
    p = torch.exp(z - want[:, None])
    p[torch.arange(n, device="cuda"), labels - tail] -= 1.0
    for got, ref in ((dw[tail:, :d], p.T @ H.double()), (dw[:1000, :d], torch.exp(-want)[None] @ H.double())):
        ref = ref.expand(got.shape)
        assert float((got.double() - ref).norm()) <= 2.0 ** -8 * float(ref.norm())
    if pitch > d:
        assert (dw[:, d:] == 7.0).all()
