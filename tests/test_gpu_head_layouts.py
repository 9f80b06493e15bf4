"""The head's gradients in matrices of every alignment: rows on 16-byte boundaries whose width is no whole number of them (what
lies between the rows belongs to others), rows off them, narrow ones; the hidden states' gradient stored directly and through
sums."""
import math

import pytest
import torch

from paper_2312_17530_b200 import binding
from test_gpu_head import TYPES, label_want, operand, run_labels, run_top

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


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,d,k", [(50, 700, 72, 9), (300, 3000, 136, 80)])
def test_what_is_masked_is_not_read(kind, n, v, d, k):
    """Logits of left-out entries and gradients of tokens without a loss may be anything: the same bits as with zeros there."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    dtype = TYPES[kind]
    H, W = operand(gen, n, d, dtype), operand(gen, v, d, dtype, 0, 2 / math.sqrt(d))
    index = torch.rand(n, v, generator=gen, device="cuda").argsort(1)[:, :k].contiguous()
    index[torch.rand(n, k, generator=gen, device="cuda") < 0.3] = -1
    index[::7] = -1
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
    labels[::7] = -100
    logit, g = torch.randn(n, k, generator=gen, device="cuda"), torch.rand(n, generator=gen, device="cuda")
    out = []
    for junk in (0.0, float("nan"), float("inf"), float("-inf"), torch.finfo(torch.float32).min):
        bad_logit, bad_g = torch.where(index < 0, junk, logit), g.clone()
        bad_g[::7] = junk
        dh, dw = [torch.empty_like(H) for _ in range(2)], [torch.empty_like(W) for _ in range(2)]
        a = run_labels(H, W, labels, bad_g, dh[0], dw[0])
        b = run_top(H, W, index, bad_logit, 2.0, bad_g, dh[1], dw[1])
        out.append([t.clone() for t in (*a, *b, *dh, *dw)])
        assert all(torch.equal(s, t) for s, t in zip(out[0], out[-1]))
        assert all(torch.isfinite(t).all() for t in out[-1])
