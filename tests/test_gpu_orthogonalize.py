"""Orthogonalised update against the polynomials in binary64.

Tolerances, derived before the first run.  The operator documents its roundings: Y in two binary16 planes of which a product
takes the first (or both), A and B in one (or two), products' sums in binary32.  `rounded` makes exactly these
roundings in binary64; how far that is from the formula, t (2-norm), is what they cost on this input, with whatever the polynomials
make of it.  The kernel's differs from it by binary32's sums (2^-24 a step of 16 terms, against 2^-12 a rounding: under a
tenth for up to 8192 terms) and by roundings that fall to the other side, each as large as the ones in t: 2 t.  With 22-bit operands the
sums are what is left: 2^-23 for each 16 terms of |A| entries, at most (K / 16) 2^-23, which the steps enlarge as they do the
roundings, by t / 2^-12 of the single product's t at most.  The result's own rounding, u, is added.
"""
import math

import pytest
import torch

from paper_2312_17530_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
COEF = binding.ORTHOGONAL_COEFFICIENTS


def half(x, scale):
    return (x * scale).half().double() / scale


def steps(x, coef, eps, products=0):
    """The formula; products = 1 or 3: with the operands' roundings of one product or three."""
    y = x.double()
    tall = y.shape[-2] > y.shape[-1]
    y = y.mT if tall else y
    y = y / (torch.linalg.matrix_norm(y)[..., None, None] + eps)

    def two(v, scale):
        hi = half(v, scale)
        return hi, half(v - hi, scale)

    def mul(a, b):  # of pairs
        if not products:
            return sum(a) @ sum(b)
        return a[0] @ b[0] + (a[0] @ b[1] + a[1] @ b[0] if products == 3 else 0)

    def plane(v, scale):
        if not products:
            return v, torch.zeros_like(v)
        hi, lo = two(v, scale)
        return (hi, lo) if products == 3 else (hi, torch.zeros_like(hi))

    for a, b, c in coef:
        yy = two(y, 4096.0) if products else (y, torch.zeros_like(y))
        A = plane(mul(yy, tuple(v.mT for v in yy)), 8192.0)
        B = plane(b * sum(A) + c * mul(A, A), 8192.0)
        y = a * sum(yy) + mul(B, yy)
    return y.mT if tall else y


def limits(x, out_dtype, coef=COEF, eps=1e-7):
    """(wanted, how far off in the 2-norm)"""
    want = steps(x, coef, eps)
    one = torch.linalg.matrix_norm(steps(x, coef, eps, 1) - want)
    side, long = min(x.shape[-2:]), max(x.shape[-2:])
    t = one
    if out_dtype == torch.float16 or side <= 256:
        t = torch.linalg.matrix_norm(steps(x, coef, eps, 3) - want) + one * 2.0 ** 12 * 2.0 ** -23 * (3 * long / 16 + 1)
    return want, 2 * t


def near(got, want, t, what=""):
    u = UNIT[got.dtype]
    d = got.double() - want
    # rounding: half a step of each value
    over = (d.abs() - u * want.abs() - TINY[got.dtype]).clamp(min=0)
    assert torch.isfinite(d).all(), what
    assert (torch.linalg.matrix_norm(over) <= t).all(), (what, torch.linalg.matrix_norm(over) / t)
    # no part of the matrix has more than its share: a block of 32 x 32, or what there is of it
    m, n = d.shape[-2:]
    pad = torch.nn.functional.pad(over, (0, -n % 32, 0, -m % 32))
    blocks = pad.unflatten(-1, (-1, 32)).unflatten(-3, (-1, 32)).square().sum((-1, -3)).sqrt()
    share = math.sqrt(min(1.0, 1024 / (m * n)))
    assert (blocks <= (6 * share) * t[..., None, None] + 1e-12).all(), (what, float((blocks.amax((-1, -2)) / t).max()), share)


def gradient(gen, shape, kind="noise"):
    g = torch.randn(*shape, generator=gen, device="cuda")
    if kind == "low":
        r = max(1, min(shape[-2:]) // 16)
        g = 0.1 * g + torch.randn(*shape[:-1], r, generator=gen, device="cuda") @ torch.randn(
            *shape[:-2], r, shape[-1], generator=gen, device="cuda") / math.sqrt(r)
    return g


def place(x, dtype, pitch=0, offset=0):
    """x with a row pitch and a start that need not be aligned; (view, buffer)"""
    *n, rows, cols = x.shape
    n = n[0] if n else 1
    pitch = pitch or cols
    buf = torch.full((offset + n * rows * pitch,), 7.0, dtype=dtype, device="cuda")
    view = buf[offset:].view(n, rows, pitch)[:, :, :cols]
    view = view if x.dim() == 3 else view[0]
    view.copy_(x.to(dtype))
    return view, buf


def run(x, out_dtype, coef=COEF, eps=1e-7, pitch=0, offset=0):
    out, buf = place(torch.zeros_like(x), out_dtype, pitch, offset)
    out.fill_(5.0)
    around = buf.clone()
    n, rows, cols = x.shape if x.dim() == 3 else (1, *x.shape)
    ws = torch.full((binding.orthogonalize_workspace_bytes(n, rows, cols, out_dtype),), 255, dtype=torch.uint8, device="cuda")
    binding.orthogonalize(x, out, ws, coef, eps)
    assert binding.operator_status() == 0
    got = out.clone()
    out.fill_(5.0)
    assert torch.equal(buf, around)
    return got


SHAPES = [(1, 1), (1, 7), (7, 1), (5, 3), (1, 300), (16, 64), (64, 64), (33, 65), (100, 257), (257, 100), (256, 256), (300, 300),
          (513, 1000), (1000, 513), (777, 1501), (260, 4100), (4100, 260), (100, 9000), (9000, 100), (1030, 1030)]


@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("m,n", SHAPES)
def test_shapes(m, n, out):
    gen = torch.Generator(device="cuda").manual_seed(m * 10007 + n)
    for kind, values, pitch, offset in (("f32", "low", 0, 0), ("bf16", "noise", n + 3, 1), ("f16", "low", (n + 15) // 8 * 8, 8)):
        x, _ = place(gradient(gen, (m, n), values), TYPES[kind], pitch, offset)
        want, t = limits(x, TYPES[out])
        near(run(x, TYPES[out], pitch=pitch, offset=offset), want, t, (kind, values))


@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("b,m,n", [(2, 1, 1), (3, 70, 130), (5, 300, 280), (40, 30, 20), (3, 257, 700), (3, 700, 257), (2, 1030, 300)])
def test_stacks(b, m, n, out):
    gen = torch.Generator(device="cuda").manual_seed(b * m + n)
    scale = torch.logspace(-6, 3, b, device="cuda")[:, None, None]
    for pitch, offset in ((0, 0), (n + 1, 3)):
        x, _ = place(gradient(gen, (b, m, n), "low") * scale, torch.float32, pitch, offset)
        want, t = limits(x, TYPES[out])
        near(run(x, TYPES[out], pitch=pitch, offset=offset), want, t)
    # matrices interleaved row by row, and the same ones alone
    x = gradient(gen, (m, b, n)).transpose(0, 1)
    got = torch.empty(m, b, n, dtype=TYPES[out], device="cuda").transpose(0, 1)
    ws = torch.empty(binding.orthogonalize_workspace_bytes(b, m, n, TYPES[out]), dtype=torch.uint8, device="cuda")
    binding.orthogonalize(x, got, ws)
    near(got, *limits(x, TYPES[out]))


def test_large():
    gen = torch.Generator(device="cuda").manual_seed(3)
    for m, n in ((2048, 2100), (20000, 600), (600, 20000)):
        x = gradient(gen, (m, n), "low").bfloat16()
        near(run(x, torch.bfloat16), *limits(x, torch.bfloat16))


@pytest.mark.parametrize("m,n", [(40, 90), (90, 40), (400, 300)])
def test_scale_of_the_input_does_not_matter(m, n):
    """The norm is taken in binary64: neither squares nor scales leave the range.  Powers of two change no bit of the result
    where eps is 0, except that binary32's own subnormal numbers have fewer digits."""
    gen = torch.Generator(device="cuda").manual_seed(m)
    x = gradient(gen, (m, n))
    want = run(x, torch.bfloat16, eps=0.0)
    for power in (-90, -60, 60, 120):
        assert torch.equal(run(x * 2.0 ** power, torch.bfloat16, eps=0.0), want)
    eps = float(torch.linalg.matrix_norm(x.double()))
    near(run(x, torch.float16, eps=eps), *limits(x, torch.float16, eps=eps))


@pytest.mark.parametrize("m,n", [(40, 90), (700, 300)])
def test_zeros_and_what_is_not_finite(m, n):
    x = torch.zeros(3, m, n, device="cuda")
    for eps in (0.0, 1e-7):
        assert (run(x, torch.bfloat16, eps=eps) == 0).all()
    x[1] = torch.randn(m, n, device="cuda")
    for bad in (float("nan"), float("inf")):
        x[2] = torch.randn(m, n, device="cuda")
        x[2, m - 1, 3] = bad
        got = run(x, torch.bfloat16)
        assert (got[0] == 0).all() and torch.isnan(got[2]).all()
        near(got[1], *limits(x[1], torch.bfloat16))


@pytest.mark.parametrize("m,n", [(64, 64), (300, 500), (500, 300)])
def test_one_value_per_row(m, n):
    """Permuted diagonal matrices: entries as large as they can be, known results."""
    k = min(m, n)
    x = torch.zeros(m, n, device="cuda")
    s = torch.linspace(0.01, 1.0, k, device="cuda")
    x[torch.randperm(m, device="cuda")[:k], torch.randperm(n, device="cuda")[:k]] = s
    want, t = limits(x, torch.float16)
    near(run(x, torch.float16), want, t + 1e-9)
    x = torch.zeros(m, n, device="cuda")
    x[m - 1, n - 1] = -3.0                           # a single one: its singular value is 1 throughout
    v = 1.0
    for a, b, c in COEF:
        v = v * (a + v * v * (b + v * v * c))
    got = run(x, torch.bfloat16).double()
    assert abs(float(got[m - 1, n - 1]) + v) <= 2.0 ** -8 * abs(v) + 2.0 ** -9
    got[m - 1, n - 1] = 0
    assert (got == 0).all()


@pytest.mark.parametrize("m,n,out", [(200, 500, "bf16"), (500, 300, "bf16"), (300, 300, "f16")])
def test_other_coefficients(m, n, out):
    """The cubic that converges: the result's shorter side is orthonormal."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    u, _, v = torch.linalg.svd(gradient(gen, (m, n)), full_matrices=False)
    x = (u * torch.linspace(0.2, 1.0, min(m, n), device="cuda")) @ v
    coef = ((1.5, -0.5, 0.0),) * 20
    got = run(x, TYPES[out], coef)
    near(got, *limits(x, TYPES[out], coef))
    g = got.double() if m <= n else got.double().mT
    # 2^-8 a value, of which a row's product has n (min(m, n) of them at random signs): their root mean square twice, for both factors
    off = g @ g.mT - torch.eye(min(m, n), device="cuda")
    assert float(off.abs().max()) <= 8 * UNIT[TYPES[out]]
    one = ((2.0, -1.5, 0.5),)
    near(run(x, TYPES[out], one), *limits(x, TYPES[out], one))


@pytest.mark.parametrize("b,m,n", [(1, 300, 200), (1, 513, 2000), (4, 100, 300)])
def test_same_bits_in_a_graph_and_on_another_stream(b, m, n):
    gen = torch.Generator(device="cuda").manual_seed(m)
    x = gradient(gen, (b, m, n))
    want = run(x, torch.bfloat16)
    ws = [torch.empty(binding.orthogonalize_workspace_bytes(b, m, n, torch.bfloat16), dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [torch.zeros_like(want) for _ in range(2)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        binding.orthogonalize(x, out[0], ws[0])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
        with torch.cuda.stream(side):
            binding.orthogonalize(x, out[1], ws[1])
    torch.cuda.synchronize()
    assert torch.equal(out[0], want) and torch.equal(out[1], want)
    assert binding.operator_status() == 0


def test_nothing_to_do():
    for shape in ((0, 5), (5, 0), (0, 3, 4), (3, 0, 4)):
        x = torch.empty(*shape, device="cuda")
        out = torch.empty(*shape, dtype=torch.bfloat16, device="cuda")
        binding.orthogonalize(x, out, torch.empty(256, dtype=torch.uint8, device="cuda"))
