"""The vocabulary head's loss and distillation from top logits, against the formulas in binary64.

Tolerances, written down before the first run (u: half the spacing of the operands' type, 2^-8 or 2^-11):
  z      the products are exact in binary32, their sums run over K/16 steps of 16 terms in the tensor core, each
         step off by at most 2^-23 of what it adds up: ez = (d/16 + 16) 2^-23 |h| |W|^T.
  lse    max ez / T for the logits; 2^-20 (1 + |lse|) for the exponentials (two units of the last place, and the
         argument's rounding), the logarithm and the change of base; the sum's chain of 128 + parts/8 additions.
  loss   lse's, plus ez / T at the targets, plus 2^-21 of the terms' sizes, times T^2.
  dz     u |dz| for the 16-bit operand (binary16: 2^-38 of the largest gradient for its subnormals), and the
         probability's own error: p |g| T (ez / T + lse's + 2^-20).
  dh,dW  dz's error through the other factor, (K/16 + 16 + pieces) 2^-23 of the absolute products, u of the result.
Sizes of the whole (2-norms): dz's rounding and the output's, each at most u in every term and independent, so u
relative suffices for random signs (sqrt(2/3) u is expected), plus half the spacing of the output's subnormals.
"""
import math

import pytest
import torch

from paper_2312_17530_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
F64 = torch.float64


def operand(gen, n, d, dtype, extra=0, scale=1.0):
    """n x d values in rows that start on 16-byte boundaries, NaN beyond the width."""
    pitch = (d + 7) // 8 * 8 + extra
    buf = torch.full((n, pitch), float("nan"), dtype=dtype, device="cuda")
    buf[:, :d] = (torch.randn(n, d, generator=gen, device="cuda") * scale).to(dtype)
    return buf[:, :d]


def output(n, d, dtype, pitch, offset=0):
    return torch.full((offset + n * pitch,), 7.0, dtype=dtype, device="cuda")[offset:].view(n, pitch)[:, :d]


def untouched(t, n, d, pitch, offset=0):
    inside = torch.zeros_like(t._base, dtype=torch.bool)
    inside[offset:].view(n, pitch)[:, :d] = True
    return bool((t._base[~inside] == 7.0).all())


def workspace(n, v, d, k=1):
    return torch.full((binding.head_workspace_bytes(n, v, d, k),), 0xFF, dtype=torch.uint8, device="cuda")  # NaNs


class Want:
    """loss, lse and gradients by the formulas, with their tolerances.  target: dense n x v; has: rows with a loss."""

    def __init__(self, H, W, target, has, own_entropy, T=1.0):
        self.H, self.W, self.T, self.target, self.has = H.double(), W.double(), T, target, has
        n, v, d = H.shape[0], W.shape[0], H.shape[1]
        z = self.H @ self.W.T
        self.ez = (d / 16 + 16) * 2.0 ** -23 * (self.H.abs() @ self.W.abs().T)
        self.lse = torch.logsumexp(z / T, 1)
        self.p = torch.exp(z / T - self.lse[:, None])
        parts = 2 * -(-v // 256)
        self.lse_tol = self.ez.amax(1) / T + 2.0 ** -20 * (1 + self.lse.abs()) + (144 + parts / 8) * 2.0 ** -24
        mass = target.sum(1)
        cross = (target * (self.lse[:, None] - z / T)).sum(1)
        self.loss = torch.where(has, T * T * (own_entropy + cross), torch.zeros_like(cross))
        terms = (target * (z.abs() / T)).sum(1) + mass * self.lse.abs() + own_entropy.abs()
        self.loss_tol = T * T * (mass * self.lse_tol + (target * self.ez).sum(1) / T + 2.0 ** -21 * (1 + terms))

    def check_forward(self, loss, lse):
        assert ((lse.double() - self.lse).abs() <= self.lse_tol).all()
        assert ((loss.double() - self.loss).abs() <= self.loss_tol).all()
        assert (loss[~self.has] == 0).all()

    def check_backward(self, g, dh, dw, dtype, pieces):
        n, v, d = self.H.shape[0], self.W.shape[0], self.H.shape[1]
        u = UNIT[dtype]
        gt = torch.where(self.has, g.double() * self.T, torch.zeros_like(self.lse))
        dz = gt[:, None] * (self.p - self.target)
        small = float(gt.abs().max()) * 2.0 ** -38 if dtype == torch.float16 else 0.0
        # the difference p - target is taken on rounded numbers: both count
        edz = u * dz.abs() + small + gt.abs()[:, None] * (
            self.p * (self.ez / self.T + self.lse_tol[:, None] + 2.0 ** -20) + 2.0 ** -22 * self.target)
        for got, ref, other, err, chain in ((dh, dz @ self.W, self.W, edz @ self.W.abs(), v),
                                            (dw, dz.T @ self.H, self.H, edz.T @ self.H.abs(), n)):
            size = dz.abs() @ other.abs() if got is dh else dz.abs().T @ other.abs()
            tol = err + (chain / 16 + 16 + pieces) * 2.0 ** -23 * size + UNIT[got.dtype] * ref.abs() + TINY[got.dtype]
            assert torch.isfinite(got).all()
            assert ((got.double() - ref).abs() <= tol).all(), float(((got.double() - ref).abs() / tol).max())
            if ref.norm() > 0 and min(n, v, d) >= 32:
                assert float((got.double() - ref).norm()) <= u * float(ref.norm()) + TINY[got.dtype] * got.numel() ** 0.5
        assert (dh[~self.has] == 0).all()


def label_want(H, W, labels):
    has = labels >= 0
    target = torch.zeros(H.shape[0], W.shape[0], dtype=F64, device="cuda")
    target.scatter_(1, labels.clamp(min=0)[:, None], has.double()[:, None])
    return Want(H, W, target, has, torch.zeros(H.shape[0], dtype=F64, device="cuda"))


def top_want(H, W, index, logit, T):
    u = (logit.double() / T).masked_fill(index < 0, -math.inf)
    has = u.amax(1) > -math.inf
    q = torch.where(has[:, None], torch.softmax(torch.where(has[:, None], u, torch.zeros_like(u)), 1), torch.zeros_like(u))
    entropy = torch.where(q > 0, q * q.clamp(min=1e-300).log(), torch.zeros_like(q)).sum(1)
    target = torch.zeros(H.shape[0], W.shape[0], dtype=F64, device="cuda")
    target.scatter_add_(1, index.clamp(min=0), q)
    return Want(H, W, target, has, entropy, T)


def run_labels(H, W, labels, g, dh, dw):
    n, d, v = H.shape[0], H.shape[1], W.shape[0]
    loss, lse = torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
    ws = workspace(n, v, d)
    binding.head_loss_forward(H, W, labels, loss, lse, ws)
    ws.fill_(0xFF)  # nothing in it has to survive between the calls
    binding.head_loss_backward(H, W, labels, lse, g, dh, dw, ws)
    assert binding.operator_status() == 0
    return loss, lse


def run_top(H, W, index, logit, T, g, dh, dw):
    n, d, v, k = H.shape[0], H.shape[1], W.shape[0], index.shape[1]
    loss, lse = torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
    ws = workspace(n, v, d, k)
    binding.head_distill_forward(H, W, index, logit, T, loss, lse, ws)
    ws.fill_(0xFF)
    binding.head_distill_backward(H, W, index, logit, T, lse, g, dh, dw, ws)
    assert binding.operator_status() == 0
    return loss, lse


SIZES = [(1, 1, 1), (1, 2, 7), (2, 63, 8), (3, 64, 16), (5, 65, 63), (1, 1000, 64), (127, 127, 65), (128, 128, 64), (129, 129, 72),
         (255, 255, 128), (256, 256, 64), (257, 257, 136), (300, 1000, 264), (64, 5001, 520), (1023, 513, 1000), (1100, 3000, 96)]


def pieces_of(n, v):
    most = max(2048, (64 << 20) // (2 * n) // 256 * 256)
    return -(-v // most)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,d", SIZES)
def test_labels(kind, n, v, d):
    gen = torch.Generator(device="cuda").manual_seed(n * 7919 + v * 31 + d)
    dtype = TYPES[kind]
    for extra, grads, pitch, offset in ((0, dtype, d, 0), (8, dtype, d + 3, 1), (24, torch.float32, d + 4, 0)):
        H, W = operand(gen, n, d, dtype, extra), operand(gen, v, d, dtype, extra, 2 / math.sqrt(d))
        labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
        labels[torch.rand(n, generator=gen, device="cuda") < 0.2] = -100
        g = torch.rand(n, generator=gen, device="cuda") * (1e-3 if extra else 1.0)
        dh, dw = output(n, d, dtype, pitch, offset), output(v, d, grads, pitch, offset)
        loss, lse = run_labels(H, W, labels, g, dh, dw)
        want = label_want(H, W, labels)
        want.check_forward(loss, lse)
        want.check_backward(g, dh, dw, dtype, pieces_of(n, v))
        assert untouched(dh, n, d, pitch, offset) and untouched(dw, v, d, pitch, offset)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,d,k,T", [(1, 1, 1, 1, 1.0), (1, 50, 8, 3, 2.0), (5, 129, 63, 33, 0.5), (130, 257, 72, 64, 3.0),
                                       (300, 1000, 264, 5, 2.0), (64, 5001, 520, 200, 1.0), (3, 1500, 64, 1024, 4.0)])
def test_top_logits(kind, n, v, d, k, T):
    gen = torch.Generator(device="cuda").manual_seed(n * 7919 + v * 31 + d + k)
    dtype = TYPES[kind]
    for top, extra in (("f32", 0), (kind, 8)):
        H, W = operand(gen, n, d, dtype, extra), operand(gen, v, d, dtype, extra, 2 / math.sqrt(d))
        index = torch.rand(n, v, generator=gen, device="cuda").argsort(1)[:, :k] if k <= v else None
        logit = operand(gen, n, k, TYPES[top], extra, 3.0)
        index = torch.nn.functional.pad(index, (0, extra), value=1 << 40)[:, :k]   # a row stride, bad values beyond
        index[torch.rand(n, k, generator=gen, device="cuda") < 0.1] = -1
        if n > 2:
            index[1] = -1                              # no entry at all
            logit[2, 0] = -math.inf                    # an entry of no weight
        if n > 4 and k > 2:
            index[3, 1] = index[3, 0]                  # the same entry twice
            logit[4, :2] = torch.finfo(logit.dtype).min
        g = torch.rand(n, generator=gen, device="cuda")
        dh, dw = output(n, d, dtype, d), output(v, d, dtype, d)
        loss, lse = run_top(H, W, index, logit, T, g, dh, dw)
        want = top_want(H, W, index, logit, T)
        want.check_forward(loss, lse)
        want.check_backward(g, dh, dw, dtype, pieces_of(n, v))


@pytest.mark.parametrize("n,v,d,k", [(8200, 9001, 72, 0), (16500, 5000, 24, 7)])
def test_several_pieces_of_the_vocabulary(n, v, d, k):
    assert pieces_of(n, v) == 3
    gen = torch.Generator(device="cuda").manual_seed(n)
    H, W = operand(gen, n, d, torch.bfloat16), operand(gen, v, d, torch.bfloat16, 0, 2 / math.sqrt(d))
    g = torch.rand(n, generator=gen, device="cuda") / n
    dh, dw = output(n, d, torch.bfloat16, d), output(v, d, torch.bfloat16, d)
    if k:
        index = torch.randint(0, v, (n, k), generator=gen, device="cuda")
        logit = torch.randn(n, k, generator=gen, device="cuda")
        loss, lse = run_top(H, W, index, logit, 2.0, g, dh, dw)
        want = top_want(H, W, index, logit, 2.0)
    else:
        labels = torch.randint(-1, v, (n,), generator=gen, device="cuda")
        loss, lse = run_labels(H, W, labels, g, dh, dw)
        want = label_want(H, W, labels)
    want.check_forward(loss, lse)
    want.check_backward(g, dh, dw, torch.bfloat16, 3)


def test_labels_and_one_top_logit_agree():
    """A teacher with one entry is a label: the same loss and gradients, bit for bit, at T = 1."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    n, v, d = 70, 777, 80
    H, W = operand(gen, n, d, torch.bfloat16), operand(gen, v, d, torch.bfloat16)
    labels = torch.randint(-1, v, (n,), generator=gen, device="cuda")
    g = torch.rand(n, generator=gen, device="cuda")
    a, b = (output(n, d, torch.bfloat16, d), output(v, d, torch.bfloat16, d)), (output(n, d, torch.bfloat16, d), output(v, d, torch.bfloat16, d))
    loss, lse = run_labels(H, W, labels, g, *a)
    loss2, lse2 = run_top(H, W, labels[:, None].contiguous(), torch.randn(n, 1, device="cuda"), 1.0, g, *b)
    assert torch.equal(lse, lse2) and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert ((loss - loss2).abs() <= 2.0 ** -21 * (1 + lse.abs())).all()


def test_rows_without_loss_bad_entries_and_large_logits():
    gen = torch.Generator(device="cuda").manual_seed(6)
    n, v, d = 40, 300, 64
    H, W = operand(gen, n, d, torch.bfloat16), operand(gen, v, d, torch.bfloat16)
    g = torch.rand(n, generator=gen, device="cuda")
    dh, dw = output(n, d, torch.bfloat16, d), output(v, d, torch.bfloat16, d)
    # no row has a loss
    loss, lse = run_labels(H, W, torch.full((n,), -1, device="cuda"), g, dh, dw)
    assert (loss == 0).all() and (dh == 0).all() and (dw == 0).all() and torch.isfinite(lse).all()
    # an entry beyond the vocabulary: loud loss, no gradient, the other rows as ever
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
    labels[3], labels[4] = v, 1 << 40
    loss, _ = run_labels(H, W, labels, g, dh, dw)
    assert torch.isnan(loss[3:5]).all() and torch.isfinite(loss[:3]).all() and torch.isfinite(loss[5:]).all()
    masked = torch.where((labels >= v), -1, labels)
    dh2, dw2 = output(n, d, torch.bfloat16, d), output(v, d, torch.bfloat16, d)
    run_labels(H, W, masked, g, dh2, dw2)
    assert torch.equal(dh, dh2) and torch.equal(dw, dw2)
    index = labels[:, None].repeat(1, 3)
    index[3, 1], index[3, 2] = 5, -1
    loss, _ = run_top(H, W, index, torch.zeros(n, 3, device="cuda"), 1.0, g, dh, dw)
    assert torch.isnan(loss[3:5]).all() and torch.isfinite(loss[5:]).all() and (dh[3:5] == 0).all()
    # an ignored row whose upstream gradient is not finite, and logits far beyond exp's range
    H2 = H.clone()
    H2[7] *= 100.0
    g[0], labels = float("inf"), masked
    labels[0] = -1
    loss, lse = run_labels(H2, W, labels, g, dh, dw)
    want = label_want(H2, W, labels)
    want.check_forward(loss, lse)
    assert (dh[0] == 0).all() and torch.isfinite(dw).all()
    # a row of hidden states that is not finite touches its own loss only
    H2[9] = float("nan")
    loss = torch.empty(n, device="cuda")
    binding.head_loss_forward(H2, W, labels, loss, None, workspace(n, v, d))
    assert torch.isnan(loss[9]) == (int(labels[9]) >= 0) and torch.isfinite(torch.cat([loss[:9], loss[10:]])).all()


@pytest.mark.parametrize("k", [0, 6])
def test_gradient_against_differences(k):
    """Hidden states on a grid of 1/64 (exact in bfloat16), moved by 1/64 along the sign of the gradient: sum g loss
    changes by twice sum |dh| / 64 from minus to plus.  The logits move by at most 0.25 at d = 64, so the cubic term is
    under 0.25^2 / 6 = 1 %; dh itself carries 0.4 % roundings."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    n, v, d = 24, 500, 64
    H = (torch.randint(-100, 101, (n, d), generator=gen, device="cuda") / 64.0).to(torch.bfloat16)
    W = operand(gen, v, d, torch.bfloat16, 0, 2 / math.sqrt(d))
    g = 0.5 + torch.rand(n, generator=gen, device="cuda")
    dh, dw = output(n, d, torch.bfloat16, d), output(v, d, torch.bfloat16, d)
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
    index = torch.rand(n, v, generator=gen, device="cuda").argsort(1)[:, :max(k, 1)].contiguous()
    logit = torch.randn(n, max(k, 1), generator=gen, device="cuda")

    def value(H):
        loss, ws = torch.empty(n, device="cuda"), workspace(n, v, d, max(k, 1))
        if k:
            binding.head_distill_forward(H, W, index, logit, 2.0, loss, None, ws)
        else:
            binding.head_loss_forward(H, W, labels, loss, None, ws)
        return float((g.double() * loss.double()).sum())

    if k:
        run_top(H, W, index, logit, 2.0, g, dh, dw)
    else:
        run_labels(H, W, labels, g, dh, dw)
    step = (dh.float().sign() / 64).to(torch.bfloat16)
    change = value(H + step) - value(H - step)
    want = 2 * float((dh.double() * step.double()).sum())
    assert want > 0 and abs(change - want) <= 0.02 * want
    # the weights' gradient through a direction in which W moves by a power of two of its own grid
    Wq = (W.float() * 64).round().div(64).to(torch.bfloat16)
    W = Wq
    (run_top(H, W, index, logit, 2.0, g, dh, dw) if k else run_labels(H, W, labels, g, dh, dw))
    step = (dw.float().sign() / 64 * (dw.float().abs() > dw.float().abs().mean())).to(torch.bfloat16)
    base = W

    def at(sign):
        nonlocal W
        W = (base.float() + sign * step.float()).to(torch.bfloat16)
        return value(H)

    change, want = at(1) - at(-1), 2 * float((dw.double() * step.double()).sum())
    assert want > 0 and abs(change - want) <= 0.2 * want


def test_repeats_other_streams_graphs_and_arena():
    gen = torch.Generator(device="cuda").manual_seed(9)
    n, v, d, k = 530, 2100, 136, 9
    H, W = operand(gen, n, d, torch.bfloat16), operand(gen, v, d, torch.bfloat16, 0, 0.2)
    labels = torch.randint(-1, v, (n,), generator=gen, device="cuda")
    index = torch.randint(0, v, (n, k), generator=gen, device="cuda")
    logit = torch.randn(n, k, generator=gen, device="cuda")
    g = torch.rand(n, generator=gen, device="cuda")
    # both heads' weight gradients into layers of a bfloat16 gradient arena
    plan = binding.Plan([(v, d, 3, 3), (v, d, 3, 3)], grad_dtype=binding.RSDGC_BF16, device=0)
    arena = torch.full((plan.info.arena_elems,), 7.0, dtype=torch.bfloat16, device="cuda")
    views = [arena[l.elem_offset:l.elem_offset + v * d].view(v, d) for l in plan.layers]
    ws = workspace(n, v, d, k)
    out = [torch.empty(n, device="cuda") for _ in range(4)] + [torch.empty(n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def step():
        binding.head_loss_forward(H, W, labels, out[0], out[1], ws)
        binding.head_loss_backward(H, W, labels, out[1], g, out[4], views[0], ws)
        binding.head_distill_forward(H, W, index, logit, 2.0, out[2], out[3], ws)
        binding.head_distill_backward(H, W, index, logit, 2.0, out[3], g, out[5], views[1], ws)

    def same(want):
        got = all(torch.equal(a, b) for a, b in zip(want, out + [arena]))
        for t in out:
            t.fill_(3.0)
        for t in views:
            t.fill_(3.0)
        return got

    step()
    want = [t.clone() for t in out + [arena]]
    assert same(want)
    step()
    assert same(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert same(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    assert same(want)
    assert binding.operator_status() == 0


def test_no_tokens():
    W = torch.randn(100, 16, device="cuda").to(torch.bfloat16)
    H, none = W[:0], torch.empty(0, device="cuda")
    labels, ws = torch.empty(0, dtype=torch.int64, device="cuda"), workspace(0, 100, 16)
    dw = output(100, 16, torch.bfloat16, 19)
    binding.head_loss_forward(H, W, labels, none, none, ws)
    binding.head_loss_backward(H, W, labels, none, none, H.clone(), dw, ws)
    assert (dw == 0).all() and untouched(dw, 100, 16, 19)


def test_refusals():
    n, v, d, k = 4, 50, 16, 3
    H, W = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(v, d, dtype=torch.bfloat16, device="cuda")
    labels, loss = torch.zeros(n, dtype=torch.int64, device="cuda"), torch.zeros(n, device="cuda")
    ws = workspace(n, v, d, k)
    good = dict(hidden=H, weight=W, labels=labels, loss=loss, lse=loss, workspace=ws)
    for bad in (dict(weight=W.half()), dict(weight=W[:, :8]), dict(labels=labels.int()), dict(labels=labels[:3]),
                dict(loss=loss.half()), dict(lse=loss[:2]), dict(workspace=ws[:100]), dict(hidden=H[0]), dict(hidden=H.t()),
                dict(labels=None), dict(labels=labels.cpu())):
        with pytest.raises(ValueError):
            binding.head_loss_forward(**{**good, **bad})
    with pytest.raises(binding.RsdgcError) as e:      # binary32 operands are not taken
        binding.head_loss_forward(**{**good, "hidden": H.float(), "weight": W.float()})
    assert e.value.code == binding.ERR_INVALID
    odd = torch.zeros(v, d + 1, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(weight=odd[:, :d]), dict(weight=odd.view(-1)[1:1 + v * d].view(v, d)), dict(workspace=torch.zeros(ws.numel() + 8, dtype=torch.uint8, device="cuda")[8:])):
        with pytest.raises(binding.RsdgcError) as e:
            binding.head_loss_forward(**{**good, **bad})
        assert e.value.code == binding.ERR_ALIGNMENT
    top, logit = torch.zeros(n, k, dtype=torch.int64, device="cuda"), torch.zeros(n, k, device="cuda")
    for T in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(binding.RsdgcError) as e:
            binding.head_distill_forward(H, W, top, logit, T, loss, loss, ws)
        assert e.value.code == binding.ERR_INVALID
    for bad in (top.int(), top[:2], top[:, :2]):
        with pytest.raises(ValueError):
            binding.head_distill_forward(H, W, bad, logit, 1.0, loss, loss, ws)
    with pytest.raises(binding.RsdgcError) as e:
        binding.head_workspace_bytes(n, v, d, 1025)
    assert e.value.code == binding.ERR_CAPACITY
    with pytest.raises(binding.RsdgcError):
        binding.head_workspace_bytes(n, 0, d)
    dh, dw = torch.zeros_like(H), torch.zeros_like(W)
    for bad in (dict(dweight=dw[:, :8]), dict(dhidden=dh.half()), dict(grad_loss=loss[:1])):
        with pytest.raises(ValueError):
            binding.head_loss_backward(**{**dict(hidden=H, weight=W, labels=labels, lse=loss, grad_loss=loss, dhidden=dh,
                                                 dweight=dw, workspace=ws), **bad})
    with pytest.raises(binding.RsdgcError) as e:      # dweight of a third type
        binding.head_loss_backward(H, W, labels, loss, loss, dh, dw.half(), ws)
    assert e.value.code == binding.ERR_INVALID
    torch.cuda.synchronize()
    assert binding.operator_status() == 0
