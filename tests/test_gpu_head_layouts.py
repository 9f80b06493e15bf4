"""The head's gradients in matrices of every alignment: rows on 16-byte boundaries whose width is no whole number of them (what
lies between the rows belongs to others), rows off them, narrow ones; the hidden states' gradient stored directly and through
sums."""
import math

import pytest
import torch

from paper_2312_17530_b200 import binding
from test_gpu_head import TYPES, label_want, operand, run_labels

pytestmark = pytest.mark.gpu


def inside_of(n, d, pitch, dtype):
    """n x d values of a larger matrix: a row above and below, columns to the right."""
    base = torch.full((n + 2, pitch), 7.0, dtype=dtype, device="cuda")
    return base, base[1:-1, :d]


def untouched(base, d):
    return bool((base[:, d:] == 7.0).all() and (base[0] == 7.0).all() and (base[-1] == 7.0).all())


@pytest.mark.parametrize("kind,grads", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("n,v,d", [(3, 50, 1), (3, 50, 2), (3, 50, 3), (40, 100, 7), (40, 100, 9), (33, 130, 61), (300, 300, 130),
                                   (140, 257, 135), (200, 520, 62), (563, 3006, 1237)])
def test_nothing_beyond_the_width_is_written(kind, grads, n, v, d):
    gen = torch.Generator(device="cuda").manual_seed(n * 31 + d)
    dtype = TYPES[kind]
    H, W = operand(gen, n, d, dtype), operand(gen, v, d, dtype, 0, 2 / math.sqrt(d))
    labels = torch.randint(-1, v, (n,), generator=gen, device="cuda")
    g = torch.rand(n, generator=gen, device="cuda")
    want = label_want(H, W, labels)
    for pitch in ((d + 7) // 8 * 8, (d + 7) // 8 * 8 + 8, d + 1, d + 2, d):
        (around_h, dh), (around_w, dw) = inside_of(n, d, pitch, dtype), inside_of(v, d, pitch, TYPES[grads])
        loss, lse = run_labels(H, W, labels, g, dh, dw)
        want.check_forward(loss, lse)
        want.check_backward(g, dh, dw, dtype, 1)
        assert untouched(around_h, d) and untouched(around_w, d)
