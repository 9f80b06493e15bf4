"""The orthogonalised update where its input is small beside eps, and the accuracy that its documentation promises.

Tolerances, derived before the first run.  `steps` makes the operator's roundings, relative to each value: operands of the products to 11 bits (or 22, with two
planes), Y to 22 bits.  How far that is from the formula, t (2-norm), is what they cost on this input; the kernel's roundings fall elsewhere, each as large: 2 t.
The products' sums are binary32 and may be cut off instead of rounded, 16 terms at a time: where all terms have one sign, a product over K terms comes out
smaller by up to (K / 16 + 1) 2^-23 (three times as many steps with two planes), in each step, and the polynomials enlarge that.  So `steps` is also computed
with each of the three products smaller by that much; what this changes is added.  What the smallest entries lose beside the largest (a plane ends 2^-37
below the norm's bound, of 2^20 entries and less: 2^-27 of the norm) is below 2^-20 of the result.
"""
import math

import pytest
import torch

from paper_2312_17530_b200 import binding
from test_gpu_orthogonalize import COEF, TYPES, gradient, near, run

pytestmark = pytest.mark.gpu


def digits(v, bits):
    m, e = torch.frexp(v)
    return torch.ldexp(torch.round(m * 2.0 ** bits), e - bits)


def steps(x, coef, eps, bits=None, smaller=(0.0, 0.0, 0.0)):
    y = x.double()
    tall = y.shape[-2] > y.shape[-1]
    y = y.mT if tall else y
    y = y / (torch.linalg.matrix_norm(y)[..., None, None] + eps)
    for a, b, c in coef:
        yy = y if bits is None else digits(y, 22)
        op = yy if bits is None else digits(yy, bits)
        A = op @ op.mT * (1 - smaller[0])
        A = A if bits is None else digits(A, bits)
        B = b * A + c * A @ A * (1 - smaller[1])
        y = a * yy + (B if bits is None else digits(B, bits)) @ op * (1 - smaller[2])
    return y.mT if tall else y


def limits(x, out_dtype, coef, eps):
    want = steps(x, coef, eps)
    side, long = sorted(x.shape[-2:])
    precise = out_dtype == torch.float16 or side <= 256
    t = 2 * torch.linalg.matrix_norm(steps(x, coef, eps, 22 if precise else 11) - want)
    for i, terms in enumerate((long, side, side)):
        smaller = [0.0, 0.0, 0.0]
        smaller[i] = ((3 if precise else 1) * terms / 16 + 1) * 2.0 ** -23
        t = t + torch.linalg.matrix_norm(steps(x, coef, eps, None, smaller) - want)
    return want, t + 2.0 ** -20 * torch.linalg.matrix_norm(want)


@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("b,m,n", [(7, 40, 90), (7, 300, 500), (2, 400, 300), (1, 5000, 300)])
def test_input_far_below_eps(b, m, n, out):
    """A gradient of 1e-13 beside an eps of 1e-7 is one of singular values 1e-6, and keeps its digits."""
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    for powers in ((-2, 2), (-14, -8), (-37, -9)):
        x = gradient(gen, (b, m, n), "low") / math.sqrt(m * n) * torch.logspace(*powers, b, device="cuda")[:, None, None]
        near(run(x, TYPES[out]), *limits(x, TYPES[out], COEF, 1e-7))
    # many steps: small values grow until they are ordinary ones
    coef = ((1.5, -0.5, 0.0),) * 20
    x = gradient(gen, (b, m, n)) / math.sqrt(m * n) * torch.logspace(-9, -3, b, device="cuda")[:, None, None]
    near(run(x, TYPES[out], coef, 1.0), *limits(x, TYPES[out], coef, 1.0))


@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("m,n", [(100, 300), (300, 500), (700, 400)])
def test_a_schedule_that_begins_steeply(m, n, out):
    """Its first polynomial of A is beyond what B's planes hold at their usual scale; and a second step of 29.6, with nothing to spare."""
    gen = torch.Generator(device="cuda").manual_seed(m)
    steep = tuple((a / 1.01, b / 1.01 ** 3, c / 1.01 ** 5) for a, b, c in (
        (8.2872, -23.5959, 17.3004), (4.1071, -2.9478, 0.5448), (3.9487, -2.9089, 0.5518), (3.3184, -2.4885, 0.51), (2.3007, -1.6689, 0.4188)))
    for coef in (steep, ((0.1717, 0.0, 0.0), (29.0, -990.0, 0.0))):
        for x in (gradient(gen, (m, n), "low"), torch.ones(m, n, device="cuda")):
            near(run(x, TYPES[out], coef, 0.0), *limits(x, TYPES[out], coef, 0.0))


def norm(d):
    """2-norm"""
    d = d if d.shape[0] <= d.shape[1] else d.mT
    return float(torch.linalg.eigvalsh(d @ d.mT)[-1].clamp(min=0).sqrt())


def dominant(gen, m, n, rows, factor):
    x = torch.randn(m, n, generator=gen, device="cuda")
    x[:rows] *= factor
    return x


def equal(gen, m, n):
    return torch.linalg.qr(torch.randn(m, n, generator=gen, device="cuda", dtype=torch.float64))[0].float().contiguous()


def uneven(gen, m, n):
    return torch.randn(m, n, generator=gen, device="cuda") * torch.logspace(-3, 0, m, device="cuda")[:, None]


@pytest.mark.parametrize("m,n,make", [
    (300, 300, equal), (384, 384, equal), (512, 512, lambda g, m, n: torch.eye(m, device="cuda")), (200, 200, equal), (300, 9000, uneven),
    (257, 257, uneven), (9000, 300, uneven), (200, 3000, uneven), (300, 9000, lambda g, m, n: torch.randn(m, n, generator=g, device="cuda")),
    (512, 3000, lambda g, m, n: dominant(g, m, n, 4, 100)), (512, 8000, lambda g, m, n: dominant(g, m, n, 32, 100)),
    (2048, 2048, lambda g, m, n: dominant(g, m, n, 4, 1000).mT.contiguous()), (1000, 4000, lambda g, m, n: torch.rand(m, n, generator=g, device="cuda"))])
def test_documented_accuracy(m, n, make):
    """The header's numbers, the result's rounding included; they are what was measured, rounded up, and derive from nothing else."""
    x = make(torch.Generator(device="cuda").manual_seed(m + n), m, n)
    want = steps(x, COEF, 1e-7)
    for out, limit in ((torch.float16, 0.001), (torch.bfloat16, 0.004 if min(m, n) <= 256 else 0.01)):
        got = run(x, out)
        assert norm(got.double() - want) <= limit * norm(want), out
