"""The language-model operators' host side, without a GPU: sizes, refusals of the C entry points (which come before any
device call), and the layer norm's and the losses' gradient formulas against differences in binary64."""
import math

import pytest
import torch

from paper_2312_17530_b200 import binding
from paper_2312_17530_b200.build import build_library


@pytest.fixture(scope="module")
def lib():
    build_library()
    return binding.lib()


P = 1 << 20  # a pointer that is never followed


def call(fn, order, good, **changed):
    return fn(*[{**good, **changed}[k] for k in order.split()])


NORM = "x xs w b y ys mean rstd n d t pt eps s"
NORM_GOOD = dict(x=P, xs=64, w=None, b=None, y=P, ys=64, mean=None, rstd=None, n=4, d=64, t=0, pt=0, eps=1e-5, s=None)
BACK = "dy dys x xs w mean rstd dx dxs dw db gt n d t pt ws s"
BACK_GOOD = dict(dy=P, dys=64, x=P, xs=64, w=None, mean=P, rstd=P, dx=P, dxs=64, dw=P, db=P, gt=0, n=4, d=64, t=0, pt=0, ws=P,
                 s=None)
LOSS = "h hs w ws y loss lse n v d t space s"
LOSS_GOOD = dict(h=P, hs=64, w=P, ws=64, y=P, loss=P, lse=P, n=4, v=100, d=64, t=1, space=P, s=None)
LOSSB = "h hs w ws y lse g dh dhs dw dws dwt n v d t space s"
LOSSB_GOOD = dict(h=P, hs=64, w=P, ws=64, y=P, lse=P, g=P, dh=P, dhs=64, dw=P, dws=64, dwt=1, n=4, v=100, d=64, t=1, space=P,
                  s=None)
TOP = "h hs w ws i is l ls lt k T loss lse n v d t space s"
TOP_GOOD = {"h": P, "hs": 64, "w": P, "ws": 64, "i": P, "is": 8, "l": P, "ls": 8, "lt": 0, "k": 8, "T": 2.0, "loss": P, "lse": P,
            "n": 4, "v": 100, "d": 64, "t": 1, "space": P, "s": None}


@pytest.mark.parametrize("change,code", [
    (dict(x=None), -1), (dict(y=None), -1), (dict(xs=63), -1), (dict(ys=63), -1), (dict(n=-1), -1), (dict(d=0), -1),
    (dict(t=3), -1), (dict(t=-1), -1), (dict(t=1, pt=2), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
    (dict(x=P + 2), -2), (dict(w=P + 1), -2), (dict(t=1, pt=1, y=P + 1), -2), (dict(mean=P + 2), -2), (dict(n=(1 << 30) + 1), -3),
    (dict(d=(1 << 24) + 1, xs=1 << 25, ys=1 << 25), -3)])
def test_layer_norm_forward_refuses(lib, change, code):
    assert call(lib.rsdgc_layer_norm_forward, NORM, NORM_GOOD, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(dy=None), -1), (dict(mean=None), -1), (dict(rstd=None), -1), (dict(dxs=1), -1), (dict(dx=None, dw=None, db=None), -1),
    (dict(ws=None), -1), (dict(gt=9), -1), (dict(dys=63), -1), (dict(ws=P + 8), -2), (dict(dw=P + 2), -2), (dict(dx=P + 2), -2)])
def test_layer_norm_backward_refuses(lib, change, code):
    assert call(lib.rsdgc_layer_norm_backward, BACK, BACK_GOOD, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(h=None), -1), (dict(w=None), -1), (dict(y=None), -1), (dict(loss=None), -1), (dict(space=None), -1), (dict(hs=63), -1),
    (dict(t=0), -1), (dict(t=7), -1), (dict(v=0), -1), (dict(d=0), -1), (dict(n=-5), -1), (dict(h=P + 8), -2), (dict(hs=65), -2),
    (dict(ws=68), -2), (dict(w=P + 2), -2), (dict(space=P + 16), -2), (dict(y=P + 4), -2), (dict(n=(1 << 24) + 1), -3),
    (dict(v=(1 << 28) + 1), -3), (dict(d=(1 << 20) + 1), -3)])
def test_head_loss_forward_refuses(lib, change, code):
    assert call(lib.rsdgc_head_loss_forward, LOSS, LOSS_GOOD, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(lse=None), -1), (dict(g=None), -1), (dict(dh=None), -1), (dict(dw=None), -1), (dict(dhs=63), -1), (dict(dws=63), -1),
    (dict(dwt=2), -1), (dict(dwt=5), -1), (dict(dh=P + 1), -2), (dict(dw=P + 1), -2), (dict(lse=P + 2), -2)])
def test_head_loss_backward_refuses(lib, change, code):
    assert call(lib.rsdgc_head_loss_backward, LOSSB, LOSSB_GOOD, **change) == code


@pytest.mark.parametrize("change,code", [
    ({"i": None}, -1), ({"l": None}, -1), ({"is": 7}, -1), ({"ls": 7}, -1), ({"lt": 4}, -1), ({"k": 0}, -1), ({"T": 0.0}, -1),
    ({"T": -2.0}, -1), ({"T": float("inf")}, -1), ({"T": float("nan")}, -1), ({"i": P + 4}, -2), ({"l": P + 2}, -2),
    ({"k": 1025, "is": 2000, "ls": 2000}, -3)])
def test_head_distill_refuses(lib, change, code):
    assert call(lib.rsdgc_head_distill_forward, TOP, TOP_GOOD, **change) == code


def test_nothing_to_do_succeeds_without_a_device(lib):
    assert call(lib.rsdgc_layer_norm_forward, NORM, NORM_GOOD, n=0, x=None, y=None) == 0
    assert call(lib.rsdgc_head_loss_forward, LOSS, LOSS_GOOD, n=0, h=None, y=None, loss=None, space=None) == 0


def test_workspace_sizes(lib):
    size = binding.head_workspace_bytes
    # the logits of a large head are never held: an eighth of their 16-bit size at most, and dh's sums
    n, v, d = 8192, 128000, 4096
    assert size(n, v, d) <= 2 * n * v // 8 * 2 + 4 * n * d + (1 << 26)
    # one piece of the vocabulary where it is small; every size has room for a row's partials
    assert size(1, 1, 1) < 1 << 16
    for a, b in [((5, 1000, 256), (6, 1000, 256)), ((64, 8000, 512), (64, 9000, 512))]:
        assert size(*a) <= size(*b)
    assert size(64, 8000, 512, 100) > size(64, 8000, 512, 1)
    for bad, code in [((-1, 10, 10, 1), -1), ((1, 0, 10, 1), -1), ((1, 10, 0, 1), -1), ((1, 10, 10, 0), -1),
                      ((1, 10, 10, 1025), -3), ((1 << 25, 10, 10, 1), -3)]:
        with pytest.raises(binding.RsdgcError) as e:
            size(*bad)
        assert e.value.code == code
    norm = binding.layer_norm_workspace_bytes
    assert norm(0, 8) > 0 and norm(10, 100) == 100 * norm(10, 1)
    for bad in [(-1, 8), (1, 0)]:
        with pytest.raises(binding.RsdgcError):
            norm(*bad)


def test_layer_norm_gradient_formula_against_differences():
    """The formula the kernels use, in binary64, against central differences (h = 1e-5: 1e-10 truncation and 1e-11 rounding
    for terms of unit size, of sums of 20)."""
    gen = torch.Generator().manual_seed(1)
    x, w, b, g = (torch.randn(3, 7, generator=gen, dtype=torch.float64) for _ in range(4))
    w, b = w[0], b[0]

    def value(x, w, b):
        m = x.mean(1, keepdim=True)
        r = ((x - m).square().mean(1, keepdim=True) + 1e-3) ** -0.5
        return ((x - m) * r * w + b), m, r

    _, m, r = value(x, w, b)
    xhat, gw = (x - m) * r, g * w
    dx = r * (gw - gw.mean(1, keepdim=True) - xhat * (gw * xhat).mean(1, keepdim=True))
    dw, db = (g * xhat).sum(0), g.sum(0)
    h = 1e-5
    for at, grad, put in ((x, dx, 0), (w, dw, 1), (b, db, 2)):
        for i in range(at.numel()):
            step = torch.zeros_like(at).view(-1)
            step[i] = h
            args = [[x, w, b], [x, w, b]]
            args[0][put], args[1][put] = at + step.view_as(at), at - step.view_as(at)
            diff = ((value(*args[0])[0] - value(*args[1])[0]) * g).sum() / (2 * h)
            assert abs(float(diff - grad.view(-1)[i])) < 1e-7


@pytest.mark.parametrize("T", [1.0, 2.5])
def test_head_gradient_formula_against_differences(T):
    """loss = T^2 KL(q || softmax(z / T)) with dz = g T (softmax(z / T) - q), dh = dz W, dW = dz^T h."""
    gen = torch.Generator().manual_seed(2)
    h, W, g = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((4, 5), (9, 5), (4,)))
    q = torch.zeros(4, 9, dtype=torch.float64)
    q[0, 3] = 1.0
    q[1, [1, 4, 8]] = torch.softmax(torch.randn(3, generator=gen, dtype=torch.float64), 0)
    q[3, [0, 2]] = 0.5                                   # row 2: nothing to aim at

    def value(h, W):
        logp = torch.log_softmax(h @ W.T / T, 1)
        return (g * T * T * torch.where(q > 0, q * (q.clamp(min=1e-300).log() - logp), torch.zeros_like(q)).sum(1)).sum()

    has = q.sum(1, keepdim=True)
    dz = (g * T)[:, None] * (torch.softmax(h @ W.T / T, 1) * has - q)
    step = 1e-5
    for at, grad, put in ((h, dz @ W, 0), (W, dz.T @ h, 1)):
        for i in range(at.numel()):
            e = torch.zeros_like(at).view(-1)
            e[i] = step
            e = e.view_as(at)
            diff = (value(*((at + e, W) if put == 0 else (h, at + e))) - value(*((at - e, W) if put == 0 else (h, at - e)))) / (2 * step)
            assert abs(float(diff) - float(grad.view(-1)[i])) < 1e-6
    assert math.isclose(float(has[2]), 0.0)
