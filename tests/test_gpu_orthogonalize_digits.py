"""The orthogonalised update where its input is small beside eps, and the accuracy that its documentation promises.

Tolerances, derived before the first run.  `steps` makes the operator's roundings, relative to each value: operands of the products to 11 bits (or 22, with two
planes), Y to 22 bits.  How far that is from the formula, t (2-norm), is what they cost on this input; the kernel's roundings fall elsewhere, each as large: 2 t.
binary32's sums and what the smallest entries lose beside the largest (a plane ends 2^-37 below the norm's bound, of 2^20 entries and less: 2^-27 of the
norm) add less than 2^-20 of the result for five steps, 2^-18 for twenty.
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


def steps(x, coef, eps, bits=None):
    y = x.double()
    tall = y.shape[-2] > y.shape[-1]
    y = y.mT if tall else y
    y = y / (torch.linalg.matrix_norm(y)[..., None, None] + eps)
    for a, b, c in coef:
        yy = y if bits is None else digits(y, 22)
        op = yy if bits is None else digits(yy, bits)
        A = op @ op.mT
        A = A if bits is None else digits(A, bits)
        B = b * A + c * A @ A
        y = a * yy + (B if bits is None else digits(B, bits)) @ op
    return y.mT if tall else y


def limits(x, out_dtype, coef, eps):
    want = steps(x, coef, eps)
    bits = 22 if out_dtype == torch.float16 or min(x.shape[-2:]) <= 256 else 11
    t = 2 * torch.linalg.matrix_norm(steps(x, coef, eps, bits) - want)
    return want, t + (2.0 ** -20 if len(coef) <= 5 else 2.0 ** -18) * torch.linalg.matrix_norm(want)


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
