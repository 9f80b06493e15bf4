"""Gated scan, forward and backward, against the formulas in binary64.

Tolerances, derived before the first run.  u: half the spacing of the output's type relative to the value, e = 2^-24.  Z = |gate| +
|bias|, M: the largest |x| and |first| so far.  The exponent -(gate + bias) log2(e) has three roundings (3 e Z), ex2 and rcp are
within 4 e and 2 e, the sum and the product around them within 2 e: b is off by eps = (3 Z + 16) e of itself.  A step h + b (x - h) adds 2
b M eps and two roundings, e M each; runs of 16 steps are joined by h + (L - Q h), twice at most: eight roundings per 16 steps,
and Q's own error, 3 e a step of it: 48 e b M.  So the error follows E_t = a E_{t-1} + 3 e M + b M (2 eps + 64 e), plus 16 e M for
a sequence shorter than its joins.  Backward, with A_t = |dy_t| + a A_{t+1}: D_t = a D_{t+1} + A (10 e + b eps), and the products that make
dx and dgate add their factors' relative errors and a rounding each.
"""
import pytest
import torch

from paper_2312_17530_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
E = 2.0 ** -24


def operand(gen, n, t, d, dtype, layout="batch", scale=1.0):
    """(view, its buffer): sequences first, steps first, or rows on odd places."""
    pitch, offset = (d + 3, 1) if layout == "odd" else (d + 2 + d % 2, 2) if layout == "padded" else (d, 0)
    buf = torch.full((offset + n * t * pitch,), 7.0, dtype=dtype, device="cuda")
    rows = buf[offset:]
    view = rows.view(t, n, pitch).transpose(0, 1)[:, :, :d] if layout == "steps" else rows.view(n, t, pitch)[:, :, :d]
    view.copy_((torch.randn(n, t, d, generator=gen, device="cuda") * scale).to(dtype))
    return view, buf


def reference(x, gate, bias, first, restart, lengths, dy=None, dlast=None):
    """The formulas, step by step, with the bounds above."""
    n, t, d = x.shape
    f64 = dict(dtype=torch.float64, device="cuda")
    x = x.double()
    z = gate.double() + (0 if bias is None else bias.double())
    eps = (3 * (gate.double().abs() + (0 if bias is None else bias.double().abs())) + 16) * E
    a, b = torch.sigmoid(z), torch.sigmoid(-z)
    length = torch.full((n,), t, device="cuda") if lengths is None else lengths.clamp(0, t)
    valid = (torch.arange(t, device="cuda") < length[:, None])[:, :, None]
    start = torch.zeros(n, t, 1, dtype=torch.bool, device="cuda") if restart is None else restart.bool()[:, :, None]
    h = torch.zeros(n, d, **f64) if first is None else first.double()
    M = torch.maximum(h.abs(), torch.zeros_like(h))
    err = 16 * E * h.abs()
    before, after, bound, top, off = (torch.zeros(n, t, d, **f64) for _ in range(5))
    for i in range(t):
        v = valid[:, i]
        prev, perr = torch.where(start[:, i], 0.0, h), torch.where(start[:, i], 0.0, err)
        M = torch.where(v, torch.maximum(M, x[:, i].abs()), M)
        before[:, i], off[:, i] = prev, perr
        h = torch.where(v, a[:, i] * prev + b[:, i] * x[:, i], h)
        err = torch.where(v, a[:, i] * perr + 3 * E * M + b[:, i] * M * (2 * eps[:, i] + 64 * E), err)
        after[:, i], bound[:, i], top[:, i] = h, err + 16 * E * M, M
    out = dict(valid=valid, y=after, y_tol=bound, last=h, last_tol=err + 16 * E * M)
    if dy is None:
        return out
    g = torch.zeros(n, d, **f64) if dlast is None else dlast.double()
    size, gerr = g.abs(), 16 * E * g.abs()
    dx, dz, dx_tol, dz_tol = (torch.zeros(n, t, d, **f64) for _ in range(4))
    for i in reversed(range(t)):
        v, ai, bi, ei = valid[:, i], a[:, i], b[:, i], eps[:, i]
        delta, A = g + dy[:, i].double(), size + dy[:, i].double().abs()
        D = gerr + A * 10 * E
        u = before[:, i] - x[:, i]
        dx[:, i] = torch.where(v, bi * delta, 0.0)
        dx_tol[:, i] = bi * (D + A * (ei + 4 * E))
        dz[:, i] = torch.where(v, delta * ai * bi * u, 0.0)
        # a = 1 - b: off by b eps; the state by its own bound and the joins of a block
        dz_tol[:, i] = bi * (2 * top[:, i] * (ai * D + A * (ai * ei + bi * ei + 8 * E)) + ai * A * (off[:, i] + 32 * E * top[:, i]))
        cut = start[:, i]
        g = torch.where(v, torch.where(cut, 0.0, ai * delta), g)
        size = torch.where(v, torch.where(cut, 0.0, ai * A), size)
        gerr = torch.where(v, torch.where(cut, 0.0, ai * D + A * bi * ei), gerr)
    out |= dict(dx=dx, dx_tol=dx_tol, dgate=dz, dgate_tol=dz_tol, dfirst=g, dfirst_tol=gerr + 16 * E * size, dbias=dz.sum((0, 1)),
                dbias_tol=(dz_tol * valid).sum((0, 1)) + 40 * E * dz.abs().sum((0, 1)))
    return out


def near(got, want, tol, dtype, where=None):
    limit = UNIT[dtype] * (want.abs() + tol) + TINY[dtype] + tol
    bad = ~((got.double() - want).abs() <= limit)
    if where is not None:
        bad &= where
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / limit).max()))


def call(n, t, d, kind, layout="batch", bias="same", first=True, restart=0.0, ragged=False, seed=0, grad=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1000 * n + 10 * t + d)
    dtype = TYPES[kind]
    x, _ = operand(gen, n, t, d, dtype, layout, 2.0)
    gate, _ = operand(gen, n, t, d, dtype, layout, 2.0)
    y, ybuf = operand(gen, n, t, d, dtype, layout)
    bt = None if bias is None else torch.float32 if bias == "f32" else dtype
    b = None if bt is None else (5 * torch.rand(d, generator=gen, device="cuda") - 1).to(bt)
    h0 = torch.randn(n, d, generator=gen, device="cuda") if first else None
    r = torch.rand(n, t, generator=gen, device="cuda") < restart if restart else None
    lengths = None
    if ragged:
        lengths = torch.randint(0, t + 1, (n,), generator=gen, device="cuda")
        lengths[0], lengths[-1] = 0, t + 5
    last = torch.full((n, d), 9.0, device="cuda")
    states = torch.full(binding.gated_scan_states_shape(n, t, d), 9.0, device="cuda")
    ybefore = y.clone()
    yb = ybuf.clone()
    binding.gated_scan_forward(x, gate, y, b, h0, last, r, lengths, states)
    dy, _ = operand(gen, n, t, d, dtype, layout, 0.5)
    dlast = torch.randn(n, d, generator=gen, device="cuda") if first else None
    dx, dxbuf = operand(gen, n, t, d, dtype, layout)
    dg, _ = operand(gen, n, t, d, dtype, layout)
    dxbefore, dgbefore, dxb = dx.clone(), dg.clone(), dxbuf.clone()
    dfirst, dbias = torch.full((n, d), 9.0, device="cuda"), torch.full((d,), 9.0, dtype=grad, device="cuda")
    ws = torch.full((binding.gated_scan_workspace_bytes(n, t, d),), 255, dtype=torch.uint8, device="cuda")
    binding.gated_scan_backward(dy, x, gate, states, dx, dg, b, dbias, dlast, dfirst, r, lengths, ws)
    assert binding.operator_status() == 0
    ref = reference(x, gate, b, h0, r, lengths, dy, dlast)
    v = ref["valid"].expand(n, t, d)
    near(y, ref["y"], ref["y_tol"], dtype, v)
    near(last, ref["last"], ref["last_tol"], torch.float32)
    near(dx, ref["dx"], ref["dx_tol"], dtype, v)
    near(dg, ref["dgate"], ref["dgate_tol"], dtype, v)
    near(dfirst, ref["dfirst"], ref["dfirst_tol"], torch.float32)
    near(dbias, ref["dbias"], ref["dbias_tol"], grad)
    # steps that do not exist, and what lies between the rows, stay as they were
    assert torch.equal(y[~v], ybefore[~v]) and torch.equal(dx[~v], dxbefore[~v]) and torch.equal(dg[~v], dgbefore[~v])
    y.copy_(ybefore)
    dx.copy_(dxbefore)
    assert torch.equal(ybuf, yb) and torch.equal(dxbuf, dxb)


SHAPES = [(1, 1, 1), (3, 1, 130), (3, 2, 7), (2, 15, 64), (2, 16, 64), (2, 17, 65), (1, 63, 64), (1, 64, 128), (2, 65, 130),
          (5, 129, 66), (3, 200, 1000), (1, 1000, 2), (2, 257, 63)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,t,d", SHAPES)
def test_shapes(n, t, d, kind):
    call(n, t, d, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["steps", "padded", "odd"])
@pytest.mark.parametrize("n,t,d", [(3, 70, 100), (2, 140, 129)])
def test_layouts(n, t, d, layout, kind):
    call(n, t, d, kind, layout, "f32", ragged=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("restart", [0.01, 0.3, 1.0])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("n,t,d", [(4, 1, 70), (4, 16, 64), (4, 300, 70)])
def test_restarts_and_lengths(n, t, d, ragged, restart, kind):
    call(n, t, d, kind, bias=None, first=restart < 0.1, restart=restart, ragged=ragged)


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("n,t,d", [(1, 5000, 70), (2, 3001, 64), (40, 50, 4096), (2500, 20, 60), (2600, 66, 3)])
def test_long_and_many(n, t, d, kind):
    """Clusters, warps that walk alone, CTAs with several sequences."""
    call(n, t, d, kind, restart=0.002, ragged=True, grad=TYPES[kind])


def make(n, t, d, dtype=torch.bfloat16, seed=5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x, gate, dy = (torch.randn(n, t, d, generator=gen, device="cuda").to(dtype) for _ in range(3))
    return x, gate, dy, torch.randn(n, d, generator=gen, device="cuda")


def test_step_by_step_is_the_whole():
    """A text answered token by token, the state handed on in place, gives what the whole call gives."""
    n, t, d = 3, 40, 200
    x, gate, _, h0 = make(n, t, d, torch.float32)
    y, last = torch.empty_like(x), torch.empty_like(h0)
    binding.gated_scan_forward(x, gate, y, None, h0, last)
    state, one = h0.clone(), torch.empty_like(x)
    for i in range(t):
        binding.gated_scan_forward(x[:, i:i + 1], gate[:, i:i + 1], one[:, i:i + 1], None, state, state)
    ref = reference(x, gate, None, h0, None, None)
    near(one, ref["y"], ref["y_tol"], torch.float32)
    near(state, ref["last"], ref["last_tol"], torch.float32)
    assert float((one - y).abs().max()) <= 2 * float(ref["y_tol"].max()) + 2 * E * float(y.abs().max())


@pytest.mark.parametrize("n,t,d", [(1, 4000, 64), (2, 100, 128), (40, 50, 4096)])
def test_same_bits_in_place_and_in_a_graph(n, t, d):
    x, gate, dy, h0 = make(n, t, d)
    b = torch.randn(d, device="cuda")
    ws = torch.empty(binding.gated_scan_workspace_bytes(n, t, d), dtype=torch.uint8, device="cuda")
    bufs = [dict(y=torch.zeros_like(x), dx=torch.zeros_like(x), dg=torch.zeros_like(x), state=h0.clone(), db=torch.zeros(d, device="cuda"),
                 st=torch.zeros(binding.gated_scan_states_shape(n, t, d), device="cuda")) for _ in range(2)]

    def both(o):
        binding.gated_scan_forward(x, gate, o["y"], b, o["state"], o["state"], None, None, o["st"])
        binding.gated_scan_backward(dy, x, gate, o["st"], o["dx"], o["dg"], b, o["db"], o["state"], o["state"], None, None, ws)

    both(bufs[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        both(bufs[1])
    bufs[1]["state"].copy_(h0)
    graph.replay()
    for k in bufs[0]:
        assert torch.equal(bufs[0][k], bufs[1][k]), k
    first = {k: v.clone() for k, v in bufs[0].items()}
    bufs[0]["state"].copy_(h0)
    both(bufs[0])
    assert all(torch.equal(first[k], bufs[0][k]) for k in first)
    assert binding.operator_status() == 0


def test_two_streams_at_once():
    n, t, d = 2, 3000, 256
    sets = [make(n, t, d, seed=s) for s in (1, 2)]
    want = []
    for x, gate, _, h0 in sets:
        y = torch.empty_like(x)
        binding.gated_scan_forward(x, gate, y, None, h0)
        want.append(y)
    got = [torch.empty_like(w) for w in want]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (x, gate, _, h0), y in zip(streams, sets, got):
            with torch.cuda.stream(s):
                binding.gated_scan_forward(x, gate, y, None, h0)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n,t,d", [(1, 500, 64), (1, 3000, 64), (40, 50, 4096)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_is_not_finite_ends_at_a_restart(n, t, d, bad):
    """... and reaches its own channel and sequence only; steps behind the length are not looked at."""
    x, gate, dy, _ = make(n, t, d, torch.float32)
    at, stop, end = t // 4, t // 2, t - 3
    restart = torch.zeros(n, t, dtype=torch.bool, device="cuda")
    restart[:, stop] = True
    lengths = torch.full((n,), end, device="cuda")
    clean = torch.zeros_like(x)
    binding.gated_scan_forward(x, gate, clean, None, None, None, restart, lengths)
    x2, gate2 = x.clone(), gate.clone()
    x2[0, at, 5] = bad
    x2[:, end:] = bad
    gate2[:, end:] = bad
    y, last = torch.zeros_like(x), torch.empty(n, d, device="cuda")
    states = torch.empty(binding.gated_scan_states_shape(n, t, d), device="cuda")
    binding.gated_scan_forward(x2, gate2, y, None, None, last, restart, lengths, states)
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[0, at:stop, 5] = True
    assert not torch.isfinite(y[hit]).any() and torch.equal(y[~hit], clean[~hit]) and torch.isfinite(last).all()
    dy2 = dy.clone()
    dy2[:, end:] = bad
    dy2[0, t - 5, 7] = bad
    dx, dg = torch.zeros_like(x), torch.zeros_like(x)
    binding.gated_scan_backward(dy2, x, gate2, states, dx, dg, None, None, None, None, restart, lengths)
    wrong = torch.zeros_like(hit)
    wrong[0, stop:t - 4, 7] = True
    assert not torch.isfinite(dx[wrong]).any() and torch.isfinite(dx[~wrong]).all()
    assert (dx[:, end:] == 0).all() and (dg[:, end:] == 0).all()


def test_gates_at_their_ends():
    """A gate of +-inf keeps or takes everything; the largest finite values give no NaN."""
    n, t, d = 1, 100, 64
    x, gate, dy, h0 = make(n, t, d, torch.float32)
    y, last = torch.empty_like(x), torch.empty_like(h0)
    states = torch.empty(binding.gated_scan_states_shape(n, t, d), device="cuda")
    dx, dg = torch.empty_like(x), torch.empty_like(x)
    for value, want in ((float("inf"), h0[:, None].expand_as(x)), (3e38, h0[:, None].expand_as(x)), (float("-inf"), x), (-3e38, x)):
        gate.fill_(value)
        binding.gated_scan_forward(x, gate, y, None, h0, last, None, None, states)
        assert float((y - want).abs().max()) <= 2.0 ** -22
        binding.gated_scan_backward(dy, x, gate, states, dx, dg)
        assert torch.isfinite(dx).all() and (dg.abs() <= 1e-30).all()


def test_nothing_to_do():
    d = 70
    db, ws = torch.full((d,), 9.0, device="cuda"), torch.empty(binding.gated_scan_workspace_bytes(3, 0, d) + 16, dtype=torch.uint8,
                                                                device="cuda")
    h0 = torch.randn(3, d, device="cuda")
    for dl in (h0, None):
        x = torch.empty(3, 0, d, device="cuda")
        last, df = torch.full((3, d), 9.0, device="cuda"), torch.full((3, d), 9.0, device="cuda")
        st = torch.empty(binding.gated_scan_states_shape(3, 0, d), device="cuda")
        binding.gated_scan_forward(x, x, x, None, dl, last, None, None, st)
        binding.gated_scan_backward(x, x, x, st, x, x, None, db, dl, df, None, None, ws)
        want = torch.zeros_like(h0) if dl is None else dl
        assert torch.equal(last, want) and torch.equal(df, want) and (db == 0).all()
        db.fill_(9.0)
    x = torch.empty(0, 5, d, device="cuda")
    binding.gated_scan_forward(x, x, x)
    binding.gated_scan_backward(x, x, x, torch.empty(0, 1, d, device="cuda"), x, x, None, db, None, None, None, None, ws)
    assert (db == 0).all()
