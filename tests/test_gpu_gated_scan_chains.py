"""The gated scan where the ways to deal its runs change: chains of 2 to 12 warps, clusters of 2 to 8 CTAs, warps that walk alone; rows on
and off 16-byte boundaries.  References and tolerances are those of test_gpu_gated_scan.py."""
import pytest
import torch

from paper_2312_17530_b200 import binding
from test_gpu_gated_scan import TYPES, call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["batch", "odd"])
@pytest.mark.parametrize("n,t,d", [
    (100, 250, 64),   # a chain of 12 warps (binary32 backward: 8)
    (75, 193, 70),    # the fewest sequences' groups of which each has a chain
    (3, 193, 1601),   # ... with a last group of one channel
    (200, 90, 64),    # 4 to 8 warps
    (10, 130, 2000),  # 2 and 4 warps
    (7, 700, 520),    # clusters of 2 (backward), a chain forward
    (5, 2100, 65),    # clusters of 8
    (1, 2100, 1030)])  # ... of 7 or 8 for 17 groups
@pytest.mark.parametrize("restart,ragged", [(0.0, False), (0.02, True)])
def test_chains(n, t, d, layout, kind, restart, ragged):
    call(n, t, d, kind, layout, restart=restart, ragged=ragged)


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("d", [1, 2, 3, 5, 7, 8, 9, 15, 63, 66])
@pytest.mark.parametrize("layout", ["batch", "steps", "odd"])
def test_narrow_rows(d, layout, kind):
    """Rows shorter than a piece of 16 bytes: several of them in one."""
    call(3, 37, d, kind, layout, restart=0.1, ragged=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_operands_that_lie_differently(kind):
    """One operand off 16-byte boundaries is enough for all to be read shifted, each by its own amount; gradients into an odd place."""
    n, t, d, dtype = 3, 50, 72, TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(1)

    def at(offset, pitch):
        buf = torch.zeros(offset + n * t * pitch, dtype=dtype, device="cuda")
        view = buf[offset:].view(n, t, pitch)[:, :, :d]
        view.copy_(torch.randn(n, t, d, generator=gen, device="cuda"))
        return view

    plain = [torch.randn(n, t, d, generator=gen, device="cuda").to(dtype) for _ in range(3)]
    results = []
    for places in ([(0, 72)] * 5, [(1, 73), (0, 72), (3, 75), (2, 74), (5, 77)], [(0, 80), (8, 72), (0, 72), (1, 72), (7, 73)]):
        x, gate, dy = (at(*p).copy_(v) for p, v in zip(places, plain))
        y, dgate = at(*places[3]), at(*places[4])
        states = torch.empty(binding.gated_scan_states_shape(n, t, d), device="cuda")
        binding.gated_scan_forward(x, gate, y, states=states)
        dx = torch.empty_like(plain[0])
        binding.gated_scan_backward(dy, x, gate, states, dx, dgate)
        results.append([y.clone(), dx, dgate.clone(), states])
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
    assert binding.operator_status() == 0


@pytest.mark.parametrize("n,t,d", [(1, 3000, 200), (100, 300, 64), (40, 30, 4096)])
def test_a_graph_gives_the_same_bits_as_calls(n, t, d):
    """A captured training step is replayed on new inputs; a call in between, of another shape and on another stream, changes nothing."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, gate, dy = (torch.randn(n, t, d, generator=gen, device="cuda").bfloat16() for _ in range(3))
    y, dx, dgate = (torch.empty_like(x) for _ in range(3))
    states = torch.empty(binding.gated_scan_states_shape(n, t, d), device="cuda")
    dbias = torch.empty(d, device="cuda")
    ws = torch.empty(binding.gated_scan_workspace_bytes(n, t, d), dtype=torch.uint8, device="cuda")

    def step():
        binding.gated_scan_forward(x, gate, y, states=states)
        binding.gated_scan_backward(dy, x, gate, states, dx, dgate, dbias=dbias, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(2):
        x.copy_(torch.randn(n, t, d, generator=gen, device="cuda"))
        step()
        want = [v.clone() for v in (y, dx, dgate, dbias)]
        for v in (y, dx, dgate, dbias, states):
            v.fill_(5.0)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            binding.gated_scan_forward(dy[:, :1, :33].contiguous(), dy[:, :1, :33].contiguous(), torch.empty_like(dy[:, :1, :33]).contiguous())
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, dgate, dbias)))
    assert binding.operator_status() == 0


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_strides_of_what_there_is_one_of(kind):
    """A single sequence, and a single step of each, out of tensors whose other stride is odd."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    big = torch.randn(6 * 5 * 65 + 1, generator=gen, device="cuda").to(TYPES[kind])
    whole = big[:6 * 5 * 64].view(6, 5, 64)
    one = torch.as_strided(big, (1, 5, 64), (333, 64, 1))
    last = torch.as_strided(big, (6, 1, 64), (320, 77, 1))
    results = []
    for x in (one, one.contiguous(), last, last.contiguous()):
        y, states = torch.empty(x.shape, dtype=x.dtype, device="cuda"), torch.empty(binding.gated_scan_states_shape(*x.shape), device="cuda")
        binding.gated_scan_forward(x, x, y, states=states)
        dx, dgate = torch.empty_like(y), torch.empty_like(y)
        binding.gated_scan_backward(x, x, x, states, dx, dgate)
        results.append((y, dx, dgate))
    for a, b in (results[:2], results[2:]):
        assert all(torch.equal(u, v) for u, v in zip(a, b))
    assert torch.equal(whole[:1], one) and binding.operator_status() == 0
