"""Layer norm (forward, backward, parameter gradients) against the formulas in binary64.

Tolerances, written down before the first run.  u is half the spacing of the output's type relative to the
value (2^-24, 2^-8, 2^-11: one rounding to nearest), e = 2^-24.  A row's sums are chains of at most 32 + 10
additions (32 values in a thread, five shuffles, five more across warps), so a sum of terms t is off by at most
42 e sum|t|; with the handful of roundings around it 64 e covers every term, taken on absolute values.  Rows
longer than a CTA's registers: a thread adds d / 1024 values, so the chains are d / 1024 + 10.  A column's sum
over the rows is a chain of rows / slots + slots / 16 + 8 additions, at most rows + 64.
"""
import numpy as np
import pytest
import torch

from paper_2312_17530_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
E = 2.0 ** -24


def matrix(gen, n, d, dtype, pitch=None, offset=0, scale=1.0, shift=0.0):
    """n x d values with a row pitch and a start that need not be aligned."""
    pitch = d if pitch is None else pitch
    buf = torch.full((offset + n * pitch,), 7.0, dtype=dtype, device="cuda")
    out = buf[offset:].view(n, pitch)[:, :d]
    out.copy_((torch.randn(n, d, generator=gen, device="cuda") * scale + shift).to(dtype))
    return out


def chain(d):
    return 64 + d / 1024


def reference(x, w, b, eps):
    x, w, b = (None if t is None else t.double() for t in (x, w, b))
    w = torch.ones(x.shape[1], dtype=torch.float64, device="cuda") if w is None else w
    b = torch.zeros_like(w) if b is None else b
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps) ** -0.5
    return (x - mean) * rstd * w + b, mean, rstd, w, b


def check_forward(x, w, b, eps, y, mean, rstd):
    ref, m, r, w, b = reference(x, w, b, eps)
    u, k, a = UNIT[x.dtype], chain(x.shape[1]) * E, x.double().abs()
    spread = a.mean(1, keepdim=True)
    assert ((mean.double()[:, None] - m).abs() <= k * spread + 2.0 ** -149).all()
    # 1 / sqrt(var + eps): half the relative error of var, whose terms are off by the mean's error too
    assert ((rstd.double()[:, None] - r).abs() <= r * k * (1 + r * spread)).all()
    tol = u * ref.abs() + TINY[x.dtype] + 2 * k * (w.abs() * r * (a + spread) * (1 + r * spread) + b.abs())
    assert ((y.double() - ref).abs() <= tol).all(), ((y.double() - ref).abs() / tol).max()


SHAPES = [(1, 1), (1, 7), (3, 8), (5, 31), (2, 64), (7, 255), (4, 256), (9, 1000), (3, 1001), (2, 1024), (2, 1032), (5, 4096),
          (3, 5000), (2, 8192), (2, 8200), (2, 16384), (1, 16400), (1, 33000), (700, 96), (600, 2050)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,d", SHAPES)
def test_forward(kind, n, d):
    gen = torch.Generator(device="cuda").manual_seed(n * 100003 + d)
    dtype = TYPES[kind]
    for params, pitch, offset in ((dtype, d, 0), (torch.float32, d + 8, 8), (dtype, d + 3, 1)):
        x = matrix(gen, n, d, dtype, pitch, offset, 2.0, 0.5)
        y = matrix(gen, n, d, dtype, pitch, offset)
        around = y.clone()
        w, b = matrix(gen, 1, d, params, shift=1.0)[0], matrix(gen, 1, d, params)[0]
        mean, rstd = torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
        binding.layer_norm_forward(x, w, b, y, mean, rstd, 1e-5)
        check_forward(x, w, b, 1e-5, y, mean, rstd)
        # nothing but the n x d values was written
        whole = y._base if y._base is not None else y
        inside = torch.zeros_like(whole, dtype=torch.bool)
        inside[offset:].view(n, pitch)[:, :d] = True
        assert (whole[~inside] == 7.0).all() and around.shape == y.shape
    # no parameters, no statistics, y over x
    x = matrix(gen, n, d, dtype)
    y = torch.empty_like(x)
    binding.layer_norm_forward(x, None, None, y, eps=1e-3)
    ref, _, r, _, _ = reference(x, None, None, 1e-3)
    a = x.double().abs()
    spread = a.mean(1, keepdim=True)
    tol = UNIT[dtype] * ref.abs() + TINY[dtype] + 2 * chain(d) * E * r * (a + spread) * (1 + r * spread)
    assert ((y.double() - ref).abs() <= tol).all()


def backward_reference(dy, x, w, mean, rstd):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    w = torch.ones(x.shape[1], dtype=torch.float64, device="cuda") if w is None else w.double()
    xhat, g = (x - mean) * rstd, dy * w
    return (rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)), (dy * xhat).sum(0), dy.sum(0),
            xhat, g)


@pytest.mark.parametrize("kind,grads", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("n,d", SHAPES + [(3000, 40), (1500, 520)])
def test_backward(kind, grads, n, d):
    gen = torch.Generator(device="cuda").manual_seed(n * 100003 + d)
    dtype, gtype = TYPES[kind], TYPES[grads]
    for pitch, offset in ((d, 0), (d + 8, 8), (d + 1, 1)):
        x, dy = matrix(gen, n, d, dtype, pitch, offset, 1.5, 0.3), matrix(gen, n, d, dtype, pitch, offset)
        dx = matrix(gen, n, d, dtype, pitch, offset)
        w = matrix(gen, 1, d, torch.float32 if offset == 8 else dtype, shift=1.0)[0]
        mean = x.float().mean(1)
        rstd = torch.rsqrt(x.float().var(1, unbiased=False) + 1e-5)
        dw, db = torch.full((d,), 9.0, dtype=gtype, device="cuda"), torch.full((d,), 9.0, dtype=gtype, device="cuda")
        ws = torch.empty(binding.layer_norm_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
        binding.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, ws)
        rx, rw, rb, xhat, g = backward_reference(dy, x, w, mean, rstd)
        k = chain(d) * E
        r, m = rstd.double()[:, None], mean.double()[:, None]
        loose = (x.double().abs() + m.abs()) * r            # |xhat| before the subtraction cancels
        tol = UNIT[dtype] * rx.abs() + TINY[dtype] + k * r * (
            g.abs() + g.abs().mean(1, keepdim=True) + (loose + xhat.abs()) * (g.abs() * loose).mean(1, keepdim=True))
        assert ((dx.double() - rx).abs() <= tol).all()
        kn = (n + 64) * E
        ub, tb = UNIT[gtype], TINY[gtype]
        assert ((dw.double() - rw).abs() <= ub * rw.abs() + tb + kn * (dy.double().abs() * loose).sum(0)).all()
        assert ((db.double() - rb).abs() <= ub * rb.abs() + tb + kn * dy.double().abs().sum(0)).all()
        whole = dx._base
        inside = torch.zeros_like(whole, dtype=torch.bool)
        inside[offset:].view(n, pitch)[:, :d] = True
        assert (whole[~inside] == 7.0).all()
        # each output alone, the same bits
        again = torch.empty_like(dw)
        binding.layer_norm_backward(dy, x, w, mean, rstd, dweight=again, workspace=ws)
        assert torch.equal(again, dw)
        again = torch.empty_like(dx)
        binding.layer_norm_backward(dy, x, w, mean, rstd, again)
        assert torch.equal(again, dx)


@pytest.mark.parametrize("n,d", [(3, 24), (2, 333), (4, 1500)])
def test_backward_against_differences(n, d):
    """The directional derivative of L = sum dy * y along a unit direction, by central differences of the
    binary32 forward pass.  Steps of h = 1/16 per value: the error of a central difference is h^2 / 6 times the
    third derivative along the direction, of order |L'| (rows have unit scale: 1/1000 of the terms' size), and
    the outputs' rounding, 2^-24 of them over h."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, dy = matrix(gen, n, d, torch.float32, scale=1.0), matrix(gen, n, d, torch.float32)
    w, b = matrix(gen, 1, d, torch.float32, shift=1.0)[0], matrix(gen, 1, d, torch.float32)[0]
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(binding.layer_norm_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
    binding.layer_norm_forward(x, w, b, y, mean, rstd)
    binding.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, ws)

    def value(x, w, b):
        binding.layer_norm_forward(x, w, b, y)
        return float((y.double() * dy.double()).sum())

    h = 1.0 / 16
    for at, grad, put in ((x, dx, 0), (w, dw, 1), (b, db, 2)):
        step = torch.randn(at.shape, generator=gen, device="cuda")
        step *= h / step.norm() * (at.numel() ** 0.5) / 16
        args = [x, w, b]
        plus, minus = list(args), list(args)
        plus[put], minus[put] = at + step, at - step
        got = (value(*plus) - value(*minus)) / 2
        want = float((grad.double() * (plus[put].double() - minus[put].double())).sum()) / 2
        size = float(grad.double().norm() * step.double().norm())
        assert abs(got - want) <= 2e-3 * size + 2.0 ** -22 * float((dy.double() * y.double()).abs().sum())


def test_rows_that_are_constant_huge_or_not_finite():
    d = 512
    x = torch.randn(6, d, device="cuda")
    x[0] = 3.0                      # no variance: xhat = 0, rstd = eps^-1/2
    x[1] = 1e18 * x[1]              # squares near the top of the range
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    w, b = torch.ones(d, device="cuda"), torch.full((d,), 0.25, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    binding.layer_norm_forward(x, w, b, y, mean, rstd, 1e-5)
    assert torch.equal(y[0], b) and abs(float(rstd[0]) * 1e-5 ** 0.5 - 1) < 1e-6
    for i in (1, 4, 5):             # rows do not touch one another
        check_forward(x[i:i + 1], w, b, 1e-5, y[i:i + 1], mean[i:i + 1], rstd[i:i + 1])
    assert torch.isnan(y[2]).any() and torch.isnan(y[3]).all()
    # eps = 0 on a constant row: 0 * inf, as the formula says
    binding.layer_norm_forward(x[:1], w, b, y[:1], eps=0.0)
    assert torch.isnan(y[0]).all()


def test_no_rows_other_streams_graphs_and_arena():
    d = 96
    empty = torch.empty(0, d, device="cuda")
    dw, db = torch.full((d,), 9.0, device="cuda"), torch.full((d,), 9.0, device="cuda")
    none = torch.empty(0, device="cuda")
    ws = torch.empty(binding.layer_norm_workspace_bytes(4096, d), dtype=torch.uint8, device="cuda")
    binding.layer_norm_forward(empty, None, None, torch.empty_like(empty))
    binding.layer_norm_backward(empty, empty, None, none, none, None, dw, db, ws)
    assert (dw == 0).all() and (db == 0).all()
    x, dy = torch.randn(4096, d, device="cuda"), torch.randn(4096, d, device="cuda")
    w = torch.randn(d, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(4096, device="cuda"), torch.empty(4096, device="cuda")
    dx = torch.empty_like(x)
    # the gradients written into layers of a compression plan's arena
    plan = binding.Plan([(1, d, 1, 9), (1, d, 1, 9)], device=0)
    arena = torch.full((plan.info.arena_elems,), -7.25, device="cuda")
    at = [l.elem_offset for l in plan.layers]

    def both():
        binding.layer_norm_forward(x, w, None, y, mean, rstd)
        binding.layer_norm_backward(dy, x, w, mean, rstd, dx, arena[at[0]:at[0] + d], arena[at[1]:at[1] + d], ws)

    both()
    want = [t.clone() for t in (y, dx, arena)]
    assert (arena[at[0] + d:at[1]] == -7.25).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (y, dx):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, arena)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for t in (y, dx):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, arena)))


def test_refusals():
    x, y = torch.zeros(4, 16, device="cuda"), torch.zeros(4, 16, device="cuda")
    m = torch.zeros(4, device="cuda")
    for bad in (dict(y=torch.zeros(4, 15, device="cuda")), dict(y=y.half()), dict(x=x.double()), dict(x=x.t()),
                dict(weight=torch.zeros(15, device="cuda")), dict(mean=torch.zeros(3, device="cuda")),
                dict(weight=torch.zeros(16)), dict(mean=m.half())):
        args = dict(x=x, weight=None, bias=None, y=y, mean=m)
        args.update(bad)
        with pytest.raises(ValueError):
            binding.layer_norm_forward(**args)
    for eps in (-1.0, float("nan")):
        with pytest.raises(binding.RsdgcError) as e:
            binding.layer_norm_forward(x, None, None, y, eps=eps)
        assert e.value.code == binding.ERR_INVALID
    with pytest.raises(binding.RsdgcError):     # parameters of a third type
        binding.layer_norm_forward(x.half(), torch.zeros(16, dtype=torch.bfloat16, device="cuda"), None, y.half())
    with pytest.raises(ValueError):             # no workspace
        binding.layer_norm_backward(x, x, None, m, m, None, torch.zeros(16, device="cuda"))
    with pytest.raises(binding.RsdgcError) as e:  # nothing asked for
        binding.layer_norm_backward(x, x, None, m, m)
    assert e.value.code == binding.ERR_INVALID
    L = binding.lib()
    p = x.data_ptr()
    fwd = lambda **k: L.rsdgc_layer_norm_forward(*[{**dict(zip("x xs w b y ys mean rstd n d t pt eps s".split(), (  # noqa: E731
        p, 16, None, None, y.data_ptr(), 16, None, None, 4, 16, 0, 0, 1e-5, None))), **k}[i]
        for i in "x xs w b y ys mean rstd n d t pt eps s".split()])
    assert fwd() == binding.OK
    assert fwd(x=None) == fwd(xs=15) == fwd(d=0) == fwd(n=-1) == fwd(t=3) == fwd(pt=1) == binding.ERR_INVALID
    assert fwd(x=p + 2) == binding.ERR_ALIGNMENT
    assert fwd(n=1 << 31) == fwd(d=1 << 25, xs=1 << 25, ys=1 << 25) == binding.ERR_CAPACITY
    torch.cuda.synchronize()
    assert binding.operator_status() == 0


@pytest.mark.parametrize("kind,n,d", [("f32", 40, 8500), ("f32", 301, 9001), ("f32", 300, 16400), ("f32", 77, 20485),
                                      ("f32", 9, 57346), ("bf16", 161, 16500), ("bf16", 20, 40003), ("f16", 33, 65000),
                                      ("f32", 500, 1001), ("f32", 400, 3001)])
def test_backward_of_wide_rows(kind, n, d):
    """Rows split over the CTAs of a cluster, in every phase; binary32 rows of a team each."""
    test_backward(kind, kind, n, d)
