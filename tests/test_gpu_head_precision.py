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
    H, W = (torch.zeros(r, (d + 7) // 8 * 8, dtype=TYPES[kind], device="cuda")[:, :d] for r in (n, v))
    H.copy_(torch.randn(n, d, generator=gen, device="cuda"))
    W.copy_(torch.randn(v, d, generator=gen, device="cuda") * (2 / math.sqrt(d)))
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
    g = torch.full((n,), g, device="cuda") if isinstance(g, float) else g(gen)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dh, dw = (torch.empty(r, d, dtype=t, device="cuda") for r, t in ((n, TYPES[kind]), (v, dweight_dtype or TYPES[kind])))
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


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,d", [(1, 500, 64), (1, 20000, 256), (2, 3000, 1000), (3, 700, 40), (8, 20000, 264), (31, 257, 72),
                                   (33, 5000, 128), (64, 8000, 512), (65, 1000, 63), (100, 3000, 1000), (127, 513, 520),
                                   (128, 6000, 200)])
def test_few_tokens_are_rounded_once(kind, n, v, d):
    """With few tokens a rounding of dz is not averaged out: the gradients are as near as the exact ones rounded once.  The two
    parts of dz have 16 bits together at least, the probabilities an error of 2^-20 (1 + |lse|) and the products' sums of
    (d / 16 + 16) 2^-23 of |h| |W|, 2^-15 at these sizes: 2^-14 of the norm, and 5 % for roundings that fall the other way.
    A dweight in binary32 shows the 2^-14 alone."""
    for dtype in (None, torch.float32):
        (dh, rh), (dw, rw) = gradients(kind, n, v, d, lambda gen: 0.01 + torch.rand(n, generator=gen, device="cuda"), n + v + d, dtype)
        for got, ref in ((dh, rh), (dw, rw)):
            once = float((ref.to(got.dtype).double() - ref).norm())
            assert float((got.double() - ref).norm()) <= 1.05 * once + 2.0 ** -14 * float(ref.norm())


def test_few_tokens_several_pieces():
    """Pieces of the vocabulary that are added to dhidden, in both planes."""
    n, v, d = 128, 600000, 24
    before = binding.launch_count()
    (dh, rh), (dw, rw) = gradients("bf16", n, v, d, lambda gen: 0.01 + torch.rand(n, generator=gen, device="cuda"), 5)
    # forward: tiles and their join; backward: the scale, a launch per piece and one more, dhidden's sum
    assert binding.launch_count() - before - 2 - 3 == 3
    for got, ref in ((dh, rh), (dw, rw)):
        once = float((ref.to(got.dtype).double() - ref).norm())
        assert float((got.double() - ref).norm()) <= 1.05 * once + 2.0 ** -14 * float(ref.norm())


def logits_of(H, W):
    """z of one vocabulary entry: its log-sum-exp, with 2^-22 for the change of base and back."""
    n, d = H.shape
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ws = torch.empty(binding.head_workspace_bytes(n, 1, d), dtype=torch.uint8, device="cuda")
    binding.head_loss_forward(H, W, torch.zeros(n, dtype=torch.int64, device="cuda"), loss, lse, ws)
    assert (loss.abs() <= 2.0 ** -22 * lse.abs()).all()
    return lse.double()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d", [512, 1024, 4096, 16384])
def test_logits_of_random_signs_have_no_bias(kind, d):
    """A truncated running sum loses about 0.25 2^-24 of its final value per step of 16 random terms, and the kernels put the mean
    back.  The slope of the error over the value: 0.08 2^-24 per step at most (0.25 without it, 0.5 with its sign turned).  The
    slope of 4096 rows is known to 0.01: the errors' root mean square is about that of the bias."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    H, W = (torch.randn(r, d, generator=gen, device="cuda").to(TYPES[kind]) for r in (4096, 1))
    z = (H.double() @ W.double().T)[:, 0]
    slope = float(((logits_of(H, W) - z) * z).sum() / (z * z).sum())
    assert abs(slope) <= 0.08 * 2.0 ** -24 * d / 16


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d", [1024, 16384])
@pytest.mark.parametrize("form", ["one sign", "leaning", "first columns", "last columns"])
def test_logits_of_any_growth_are_within_the_products_bound(kind, d, form):
    """(d / 16 + 16) 2^-23 of |h| |W| however the sum grows, the correction included."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    H, W = (torch.randn(r, d, generator=gen, device="cuda") for r in (512, 1))
    if form == "one sign":
        H, W = H.abs(), W.abs()
    elif form == "leaning":
        H += W
    else:
        part = slice(0, d // 8) if form == "first columns" else slice(d - d // 8, d)
        H *= 0.02
        H[:, part] += W[:, part]
    H, W = H.to(TYPES[kind]), W.to(TYPES[kind])
    z, size = (H.double() @ W.double().T)[:, 0], (H.double().abs() @ W.double().abs().T)[:, 0]
    assert ((logits_of(H, W) - z).abs() <= (d / 16 + 16) * 2.0 ** -23 * size + 2.0 ** -22 * z.abs()).all()
