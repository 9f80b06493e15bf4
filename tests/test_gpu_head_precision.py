"""How far the head's gradients are from the formula in binary64 as a whole (2-norms), where roundings do not average out.

u is half the spacing of the type relative to its values (2^-8 or 2^-11).  Rounding values of all magnitudes once leaves
about 0.42 u of their 2-norm: the spacing's root mean square, 2 u / sqrt(12), over significands between 1 and 2."""
import math

import pytest
import torch

from paper_2312_17530_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def gradients(kind, n, v, d, g, seed, dweight_dtype=None):
    """(dhidden, dweight) of the kernels and of the formula, for a head that has learnt nothing."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    H = torch.randn(n, d, generator=gen, device="cuda").to(TYPES[kind])
    W = (torch.randn(v, d, generator=gen, device="cuda") * (2 / math.sqrt(d))).to(TYPES[kind])
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
    g = torch.full((n,), g, device="cuda") if isinstance(g, float) else g(gen)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dh, dw = torch.empty_like(H), torch.empty(v, d, dtype=dweight_dtype or TYPES[kind], device="cuda")
    ws = torch.full((binding.head_workspace_bytes(n, v, d),), 0xFF, dtype=torch.uint8, device="cuda")
    binding.head_loss_forward(H, W, labels, loss, lse, ws)
    binding.head_loss_backward(H, W, labels, lse, g, dh, dw, ws)
    assert binding.operator_status() == 0
    H, W = H.double(), W.double()
    dz = torch.softmax(H @ W.T, 1)
    dz[torch.arange(n, device="cuda"), labels] -= 1.0
    dz *= g.double()[:, None]
    return (dh, dz @ W), (dw, dz.T @ H)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_equal_gradients_are_not_rounded_alike(kind):
    """The mean over the tokens: every token has the same gradient, here the worst one, just beyond a power of two.  The
    entries of dz at the labels, nearly all of it, would all be off by half a unit the same way (0.9 u of dh and dW).  Half of
    u allows the outputs' one rounding and 0.26 u besides."""
    u = UNIT[kind]
    for got, ref in gradients(kind, 512, 20000, 256, (1 + u) / 256, 3):
        assert float((got.double() - ref).norm()) <= 0.5 * u * float(ref.norm())
