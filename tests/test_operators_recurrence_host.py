"""The gated scan's and the orthogonalised update's host side, without a GPU: sizes, refusals (which come before any device call),
and the scan's gradient formulas against differences in binary64."""
import ctypes as C
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


SCAN = "x xs xt g gs gt b y ys yt first last r rs len st n t d type pt s"
SCAN_GOOD = dict(x=P, xs=640, xt=64, g=P, gs=640, gt=64, b=P, y=P, ys=640, yt=64, first=P, last=P, r=P, rs=10, len=P, st=P, n=4, t=10,
                 d=64, type=1, pt=0, s=None)
BACK = "dy dys dyt x xs xt g gs gt b st dlast dx dxs dxt dg dgs dgt db dfirst r rs len n t d type pt gradt ws s"
BACK_GOOD = dict(dy=P, dys=640, dyt=64, x=P, xs=640, xt=64, g=P, gs=640, gt=64, b=P, st=P, dlast=P, dx=P, dxs=640, dxt=64, dg=P, dgs=640,
                 dgt=64, db=P, dfirst=P, r=P, rs=10, len=P, n=4, t=10, d=64, type=1, pt=0, gradt=0, ws=P, s=None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), -1), (dict(g=None), -1), (dict(y=None), -1), (dict(xt=63), -1), (dict(gs=63), -1), (dict(yt=63), -1), (dict(ys=1), -1),
    (dict(n=-1), -1), (dict(t=-1), -1), (dict(d=0), -1), (dict(type=3), -1), (dict(type=-1), -1), (dict(type=1, pt=2), -1),
    (dict(rs=9), -1), (dict(x=P + 1), -2), (dict(y=P + 1), -2), (dict(b=P + 2), -2), (dict(first=P + 2), -2), (dict(last=P + 1), -2),
    (dict(len=P + 4), -2), (dict(st=P + 2), -2), (dict(n=(1 << 30) + 1), -3), (dict(t=(1 << 30) + 1), -3), (dict(d=(1 << 24) + 1), -3),
    (dict(n=1 << 28, d=65, xs=1 << 20, xt=65, gt=65, yt=65), -3)])
def test_scan_forward_refuses(lib, change, code):
    assert call(lib.rsdgc_gated_scan_forward, SCAN, SCAN_GOOD, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(dy=None), -1), (dict(x=None), -1), (dict(g=None), -1), (dict(st=None), -1), (dict(ws=None), -1), (dict(dxt=63), -1),
    (dict(dgs=1), -1), (dict(dyt=63), -1), (dict(dx=None, dg=None, db=None, dfirst=None), -1), (dict(gradt=3), -1), (dict(rs=9), -1),
    (dict(type=5), -1), (dict(type=2, pt=1), -1), (dict(ws=P + 8), -2), (dict(db=P + 2), -2), (dict(dx=P + 1), -2), (dict(dlast=P + 2), -2),
    (dict(dfirst=P + 2), -2), (dict(st=P + 2), -2), (dict(n=1 << 31), -3)])
def test_scan_backward_refuses(lib, change, code):
    assert call(lib.rsdgc_gated_scan_backward, BACK, BACK_GOOD, **change) == code


def test_scan_of_no_sequences_does_nothing(lib):
    nothing = {k: None for k in ("x", "g", "y", "b", "first", "last", "r", "len", "st")}
    assert call(lib.rsdgc_gated_scan_forward, SCAN, SCAN_GOOD, n=0, **nothing) == 0


def test_scan_sizes(lib):
    assert binding.gated_scan_states_shape(3, 33, 7) == (3, 3, 7) and binding.gated_scan_states_shape(2, 0, 5) == (2, 0, 5)
    size = binding.gated_scan_workspace_bytes
    # a row of sums per sequence part, or one per CTA that shares a sequence's steps: not more than eight
    for n, t, d in ((1, 1, 1), (1, 65536, 1024), (8, 4096, 4096), (5000, 20, 60), (1 << 20, 3, 64), (2, 1 << 24, 16)):
        assert 4 * d <= size(n, t, d) <= 4 * d * min(n, max(1, 16 * 148 // -(-d // 64))) * 8
    assert size(1 << 20, 3, 64) <= 1 << 20
    for bad in ((-1, 4, 4), (4, -1, 4), (4, 4, 0)):
        with pytest.raises(binding.RsdgcError):
            size(*bad)


ORTHO = "x xr xm type out outr outm outt n m k coef steps eps ws s"
COEF = (C.c_float * 3)(3.4445, -4.7750, 2.0315)
ORTHO_GOOD = dict(x=P, xr=40, xm=1200, type=0, out=P, outr=40, outm=1200, outt=1, n=2, m=30, k=40, coef=COEF, steps=1, eps=1e-7, ws=P, s=None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), -1), (dict(out=None), -1), (dict(ws=None), -1), (dict(coef=None), -1), (dict(steps=0), -1), (dict(steps=33), -1),
    (dict(xr=39), -1), (dict(outr=39), -1), (dict(xm=39), -1), (dict(outm=0), -1), (dict(type=3), -1), (dict(outt=0), -1), (dict(outt=7), -1),
    (dict(n=-1), -1), (dict(m=-1), -1), (dict(k=-2), -1), (dict(eps=-1e-9), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(x=P + 2), -2), (dict(out=P + 1), -2), (dict(ws=P + 128), -2), (dict(m=(1 << 24) + 1), -3),
    (dict(m=(1 << 15) + 1, k=(1 << 15) + 1, xr=1 << 16, outr=1 << 16), -3), (dict(n=(1 << 20) + 1), -3),
    (dict(n=1 << 20, m=1 << 14, k=1 << 14, xr=1 << 14, outr=1 << 14), -3)])
def test_orthogonalize_refuses(lib, change, code):
    assert call(lib.rsdgc_orthogonalize, ORTHO, ORTHO_GOOD, **change) == code


@pytest.mark.parametrize("coef", [(7.0, 0.0, 0.0), (2.0, 2.0, 0.0), (float("nan"), 0, 0), (1.0, float("inf"), 0), (1.0, -30.0, 8.0), (2000.0, -1999.0, 0.0)])
def test_orthogonalize_refuses_what_grows(lib, coef):
    """A singular value above 2, or the polynomial of A above 7.5."""
    assert call(lib.rsdgc_orthogonalize, ORTHO, ORTHO_GOOD, coef=(C.c_float * 3)(*coef)) == -1


def test_orthogonalize_sizes(lib):
    size = binding.orthogonalize_workspace_bytes
    for shape in ((0, 5, 5), (3, 0, 5), (3, 5, 0)):
        assert size(*shape, torch.bfloat16) == 0
    for n, m, k in ((1, 1, 1), (1, 4096, 4096), (24, 256, 1024), (1, 32000, 1024), (3, 1501, 777)):
        # two matrices of two planes, A and B of one or two, parts of A
        least = 8 * n * m * k + 4 * n * min(m, k) ** 2
        assert least <= size(n, m, k, torch.bfloat16) <= 2 * least + (64 << 20) + 8 * n * (m + k) * 8
        assert size(n, m, k, torch.bfloat16) <= size(n, m, k, torch.float16)
        assert size(n, m, k, torch.float16) % 256 == 0
    with pytest.raises(binding.RsdgcError):
        size(1, 5, 5, torch.float32)


def scan(x, gate, bias, first, restart):
    h, ys = first, []
    for t in range(x.shape[1]):
        a = torch.sigmoid(gate[:, t] + bias)
        h = a * torch.where(restart[:, t, None], 0.0, h) + (1 - a) * x[:, t]
        ys.append(h)
    return torch.stack(ys, 1), h


def test_scan_gradient_formulas_against_differences():
    gen = torch.Generator().manual_seed(3)
    n, t, d = 2, 9, 3
    x, gate, dy = (torch.randn(n, t, d, generator=gen, dtype=torch.float64) for _ in range(3))
    bias, first, dlast = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((d,), (n, d), (n, d)))
    restart = torch.rand(n, t, generator=gen) < 0.3

    def objective(x, gate, bias, first):
        y, last = scan(x, gate, bias, first, restart)
        return ((y * dy).sum() + (last * dlast).sum()).item()

    # the formulas of the header
    y, _ = scan(x, gate, bias, first, restart)
    a = torch.sigmoid(gate + bias)
    before = torch.cat([first[:, None], y[:, :-1]], 1).masked_fill(restart[:, :, None], 0.0)
    delta, dx, dgate = dlast, torch.zeros_like(x), torch.zeros_like(x)
    for i in reversed(range(t)):
        delta = delta + dy[:, i]
        dx[:, i] = (1 - a[:, i]) * delta
        dgate[:, i] = delta * a[:, i] * (1 - a[:, i]) * (before[:, i] - x[:, i])
        delta = torch.where(restart[:, i, None], 0.0, a[:, i] * delta)
    got = dict(x=dx, gate=dgate, bias=dgate.sum((0, 1)), first=delta)
    args = dict(x=x, gate=gate, bias=bias, first=first)
    step = 1e-5
    for name, grad in got.items():
        for i in range(args[name].numel()):
            side = []
            for s in (step, -step):
                moved = args[name].clone()
                moved.view(-1)[i] += s
                side.append(objective(**{**args, name: moved}))
            # third derivatives of order 1 times step^2, and 2^-53 of an objective of order 10 over the step
            assert math.isclose((side[0] - side[1]) / (2 * step), grad.reshape(-1)[i].item(), rel_tol=1e-7, abs_tol=1e-8)


def test_example_says_what_it_does_not_take():
    from paper_2312_17530_b200 import lm_step

    for bad in (dict(n_texts=-1), dict(n_texts=7), dict(update="adam")):
        with pytest.raises(ValueError):
            lm_step.run(**bad)
