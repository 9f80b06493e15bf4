"""Layer norm where the operands' rows lie differently from one another: inputs whose rows have different phases (the general
kernels), outputs whose rows have another phase than the inputs' (stored value by value by the warp's, the ring's and the
cluster's kernels), and rows wider than a cluster holds.  Tolerances are those of test_gpu_layer_norm."""
import pytest
import torch

from paper_2312_17530_b200 import binding
from test_gpu_layer_norm import E, TINY, TYPES, UNIT, backward_reference, chain, check_forward, matrix

pytestmark = pytest.mark.gpu

# (pitch beyond the width, offset) of x, dy or y, and dx: the same rows for all; inputs alike and the output shifted, against
# aligned and against shifted inputs, and by a pitch of its own; inputs that differ by an offset and by a pitch
LAYOUTS = [((0, 0), (0, 0), (0, 3)), ((3, 1), (3, 1), (0, 0)), ((0, 0), (8, 0), (1, 0)), ((8, 0), (8, 1), (8, 0)),
           ((0, 2), (3, 2), (0, 2)), ((1, 0), (2, 0), (0, 5))]


def clean(t, n, d, pitch, offset):
    """Nothing but the n x d values was written."""
    inside = torch.zeros_like(t._base, dtype=torch.bool)
    inside[offset:].view(n, pitch)[:, :d] = True
    return bool((t._base[~inside] == 7.0).all())


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,d", [(1, 5), (40, 24), (130, 100), (70, 777), (33, 1001), (90, 4100), (9, 9001), (5, 16500), (3, 33000)])
def test_forward(kind, n, d):
    gen = torch.Generator(device="cuda").manual_seed(n * 100003 + d)
    dtype = TYPES[kind]
    for (px, ox), _, (py, oy) in LAYOUTS:
        x = matrix(gen, n, d, dtype, d + px, ox, 2.0, 0.5)
        y = matrix(gen, n, d, dtype, d + py, oy)
        w, b = matrix(gen, 1, d, dtype, shift=1.0)[0], matrix(gen, 1, d, dtype)[0]
        mean, rstd = torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
        binding.layer_norm_forward(x, w, b, y, mean, rstd, 1e-5)
        check_forward(x, w, b, 1e-5, y, mean, rstd)
        assert clean(y, n, d, d + py, oy)
    assert binding.operator_status() == 0


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,d", [(1, 5), (40, 24), (130, 100), (63, 513), (64, 777), (65, 1001), (300, 1000), (90, 4100), (33, 8500),
                                 (9, 9001), (7, 16500), (20, 40003), (3, 66000)])
def test_backward(kind, n, d):
    gen = torch.Generator(device="cuda").manual_seed(n * 100003 + d)
    dtype = TYPES[kind]
    for (px, ox), (pg, og), (pd, od) in LAYOUTS:
        x, dy = matrix(gen, n, d, dtype, d + px, ox, 1.5, 0.3), matrix(gen, n, d, dtype, d + pg, og)
        dx = matrix(gen, n, d, dtype, d + pd, od)
        w = matrix(gen, 1, d, dtype, shift=1.0)[0]
        mean = x.float().mean(1)
        rstd = torch.rsqrt(x.float().var(1, unbiased=False) + 1e-5)
        dw, db = torch.full((d,), 9.0, dtype=dtype, device="cuda"), torch.full((d,), 9.0, dtype=dtype, device="cuda")
        ws = torch.full((binding.layer_norm_workspace_bytes(n, d) + 4096,), 0x41, dtype=torch.uint8, device="cuda")
        binding.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, ws[:-4096])
        assert (ws[-4096:] == 0x41).all()
        rx, rw, rb, xhat, g = backward_reference(dy, x, w, mean, rstd)
        k, kn = chain(d) * E, (n + 64) * E
        r, m = rstd.double()[:, None], mean.double()[:, None]
        loose = (x.double().abs() + m.abs()) * r
        tol = UNIT[dtype] * rx.abs() + TINY[dtype] + k * r * (
            g.abs() + g.abs().mean(1, keepdim=True) + (loose + xhat.abs()) * (g.abs() * loose).mean(1, keepdim=True))
        assert ((dx.double() - rx).abs() <= tol).all()
        ub, tb = UNIT[dtype], TINY[dtype]
        assert ((dw.double() - rw).abs() <= ub * rw.abs() + tb + kn * (dy.double().abs() * loose).sum(0)).all()
        assert ((db.double() - rb).abs() <= ub * rb.abs() + tb + kn * dy.double().abs().sum(0)).all()
        assert clean(dx, n, d, d + pd, od)
        again = torch.empty_like(dw)
        binding.layer_norm_backward(dy, x, w, mean, rstd, dweight=again, workspace=ws)
        assert torch.equal(again, dw)
    assert binding.operator_status() == 0
