"""The gated scan's digits where a gate is nearly closed: a = 1 / (1 + exp(-z)) far below 1 takes part in dgate, dfirst and dbias as a factor, and
carries the state on where x is small.

The bound is relative, term by term, derived before the first run.  e = 2^-24, Z = |gate| + |bias|.  As in test_gpu_gated_scan.py b is off by eps =
(3 Z + 16) e of itself, and so is a below 1/33, where it is formed as a product; from 1/33 on it may be 1 - b, which b's three roundings put off by 3 e
more: ea = eps + 3 e / a there.  H_t = a H_{t-1} + b |x_t| is the recurrence of the absolute values.  A step is off by ea and eps of its two terms and
four roundings of H_t at most, and what joins runs a few roundings of H more: E_t = a E_{t-1} + (ea + eps + 8 e) H_t.  Backward, A_t = |dy_t| + a_{t+1}
A_{t+1}: D_t, the error of delta_t, is e A_t and what was carried, a D + (ea + 4 e) a A; the products that make dx and dgate add their factors' relative
errors and a rounding each.  dbias: the entries' errors and 40 e of the sum of their absolute values, as there.
"""
import pytest
import torch

from paper_2312_17530_b200 import binding
from test_gpu_gated_scan import E, TYPES, near

pytestmark = pytest.mark.gpu


def reference(x, gate, bias, first, dy, dlast):
    n, t, d = x.shape
    f64 = dict(dtype=torch.float64, device="cuda")
    x, dy, zero = x.double(), dy.double(), torch.zeros(n, d, **f64)
    z = gate.double() + bias.double()
    eps = (3 * (gate.double().abs() + bias.double().abs()) + 16) * E
    a, b = torch.sigmoid(z), torch.sigmoid(-z)
    ea = eps + torch.where(a > 0.9 / 33, 3 * E / a, 0.0)
    h = zero if first is None else first.double()
    H, err = h.abs(), zero
    y, y_tol, before, size, off, dx, dx_tol, dz, dz_tol = (torch.zeros(n, t, d, **f64) for _ in range(9))
    for i in range(t):
        before[:, i], size[:, i], off[:, i] = h, H, err
        h, H = a[:, i] * h + b[:, i] * x[:, i], a[:, i] * H + b[:, i] * x[:, i].abs()
        err = a[:, i] * err + (ea[:, i] + eps[:, i] + 8 * E) * H
        y[:, i], y_tol[:, i] = h, err
    out = dict(y=y, y_tol=y_tol, last=h, last_tol=err)
    g = zero if dlast is None else dlast.double()
    G, gerr = g.abs(), zero
    for i in reversed(range(t)):
        ai, bi, ei = a[:, i], b[:, i], eps[:, i]
        delta, A = g + dy[:, i], G + dy[:, i].abs()
        D = gerr + E * A
        u, U = before[:, i] - x[:, i], size[:, i] + x[:, i].abs()
        dx[:, i], dx_tol[:, i] = bi * delta, bi * (D + A * (ei + 2 * E))
        dz[:, i] = delta * ai * bi * u
        dz_tol[:, i] = ai * bi * (D * U + A * (off[:, i] + E * U) + A * U * (ea[:, i] + ei + 6 * E))
        g, G, gerr = ai * delta, ai * A, ai * D + (ea[:, i] + 4 * E) * ai * A
    return out | dict(dx=dx, dx_tol=dx_tol, dgate=dz, dgate_tol=dz_tol, dfirst=g, dfirst_tol=gerr + 2 * E * G, dbias=dz.sum((0, 1)),
                      dbias_tol=dz_tol.sum((0, 1)) + 40 * E * dz.abs().sum((0, 1)))


def check(x, gate, bias, first, dy, dlast):
    n, t, d = x.shape
    y, dx, dgate = (torch.empty_like(x) for _ in range(3))
    last, dfirst = torch.empty(n, d, device="cuda"), torch.empty(n, d, device="cuda")
    states, dbias = torch.empty(binding.gated_scan_states_shape(n, t, d), device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(binding.gated_scan_workspace_bytes(n, t, d), dtype=torch.uint8, device="cuda")
    binding.gated_scan_forward(x, gate, y, bias, first, last, None, None, states)
    binding.gated_scan_backward(dy, x, gate, states, dx, dgate, bias, dbias, dlast, dfirst, None, None, ws)
    assert binding.operator_status() == 0
    ref = reference(x, gate, bias, first, dy, dlast)
    for name, got in dict(y=y, last=last, dx=dx, dgate=dgate, dfirst=dfirst, dbias=dbias).items():
        near(got, ref[name], ref[name + "_tol"], got.dtype)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,t,d", [(1, 1, 70), (3, 16, 64), (4, 100, 130), (40, 40, 4096)])
def test_nearly_closed_gates(n, t, d, kind):
    """Levels of -20 to 8 by channel, most of them in the bias; tokens of all sizes, some of them zeros."""
    dtype = TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(n + t + d)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    level = torch.linspace(-20, 8, d, device="cuda") if d > 1 else torch.full((1,), -14.0, device="cuda")
    x = normal(n, t, d) * 10.0 ** (3 * normal(n, t, 1).clamp(-1, 1)) * (torch.rand(n, t, d, generator=gen, device="cuda") < 0.7)
    check(x.to(dtype), normal(n, t, d).to(dtype), level.to(dtype), normal(n, d), normal(n, t, d).to(dtype), normal(n, d))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,t,d", [(100, 250, 64), (75, 193, 70), (1, 2100, 200), (3, 1700, 64)])
def test_behind_a_large_token(n, t, d, kind):
    """Chains that hand the state on ahead of their steps, and clusters: a token of 1e6 among ordinary ones, and what has decayed of it some dozens of
    steps on, by gates from open to closed and by slow channels."""
    dtype = TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(n + t + d)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    x = normal(n, t, d)
    x[:, 5::97] *= 1e6
    level = torch.linspace(-2, 9, d, device="cuda")[torch.randperm(d, generator=gen, device="cuda")]
    check(x.to(dtype), (0.3 * normal(n, t, d)).to(dtype), level.to(dtype), 1e6 * normal(n, d), normal(n, t, d).to(dtype), normal(n, d))
