"""The example with a gated scan below the norm and orthogonalised updates: it runs, repeats bit for bit, its arena holds the formulas'
gradients, and its step is the formula's."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("texts,update,rate", [(4, "sgd", 4.0), (0, "orthogonal", 0.002), (8, "orthogonal", 0.002), (1, "orthogonal", 0.002)])
def test_example_runs_and_repeats(texts, update, rate):
    from paper_2312_17530_b200 import lm_step

    args = dict(steps=6, n_tokens=240, vocab=777, width=136, n_top=7, n_texts=texts, update=update, rate=rate)
    losses = lm_step.run(**args)
    assert len(losses) == 6 and all(x == x and 0 < x < float("inf") for x in losses)
    assert lm_step.run(**args) == losses


def reference(worker, student, temperature):
    """Gradients of the worker's mean loss for the parameters that the kernels read, by automatic differentiation in binary64."""
    head, weight, bias = (t.double().requires_grad_() for t in student.views(student.shadow))
    matrix, gate_bias = (t.double().requires_grad_() for t in student.gate(student.shadow))
    x = worker.texts(worker.x).double()
    a = torch.sigmoid(x @ matrix.T + gate_bias)
    h, states = torch.zeros_like(x[:, 0]), []
    for t in range(x.shape[1]):
        h = a[:, t] * h + (1 - a[:, t]) * x[:, t]
        states.append(h)
    mixed = torch.stack(states, 1).reshape(worker.x.shape)
    hidden = torch.nn.functional.layer_norm(mixed, mixed.shape[1:], weight, bias, 1e-5)
    logits = hidden @ head.T
    hard = torch.nn.functional.cross_entropy(logits[:worker.half], worker.labels, ignore_index=-1, reduction="sum")
    p = torch.softmax(worker.top_logit.double() / temperature, 1)
    q = torch.log_softmax(logits[worker.half:] / temperature, 1).gather(1, worker.top_index)
    soft = temperature ** 2 * (p * (p.log() - q)).sum()
    ((hard + soft) / worker.x.shape[0]).backward()
    return [t.grad for t in (head, weight, bias, matrix, gate_bias)]


@pytest.mark.parametrize("texts", [1, 4])
def test_gradients_in_the_arena(texts):
    """Between a parameter and its gradient lie at most a dozen values of bfloat16 (gate, mixed, hidden, dz, dhidden, dmixed, dgate, the
    gradient, and what the norm makes of the errors before it), each off by 2^-8 of itself at most: 16 * 2^-8 of the norm."""
    from paper_2312_17530_b200 import lm_step

    teacher = torch.randn(500, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9)) * 0.4
    student = lm_step.Student(500, 64, 1, mixes=True)
    worker = lm_step.Worker(student, 96, 5, teacher, 2, texts)
    worker.arena.fill_(7.0)
    worker.gradients(2.0)
    got = [*student.views(worker.arena), *student.gate(worker.arena)]
    for g, want in zip(got, reference(worker, student, 2.0)):
        assert (g.double() - want).norm() <= 16 * 2.0 ** -8 * want.norm()
    inside = torch.zeros_like(worker.arena, dtype=torch.bool)
    for l in student.plan.layers:
        inside[l.elem_offset:l.elem_offset + l.rows * l.cols] = True
    assert (worker.arena[~inside] == 7.0).all()


def test_orthogonal_step_is_the_formula():
    """Both matrices move by rate * sqrt(longer side) * (the formula's matrix, within 0.002 of its norm and a rounding to bfloat16), the
    vectors by rate * gradient."""
    from paper_2312_17530_b200 import binding, lm_step

    student = lm_step.Student(300, 72, 4, mixes=True)
    dense = torch.randn(student.masters.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) * 1e-3
    before, gradient = student.masters.clone(), dense.clone()
    student.orthogonal_step(dense, 0.01)
    moved = [*student.views(before - student.masters), *student.gate(before - student.masters)]
    for got, g in zip(moved, [*student.views(gradient), *student.gate(gradient)]):
        if g.dim() == 1:
            # the difference of masters of order 1: two roundings of 2^-24
            assert (got.double() - 0.01 * g.double()).abs().max() <= 2.0 ** -22
            continue
        y = g.double()
        y = y / (y.norm() + 1e-7)
        for a, b, c in binding.ORTHOGONAL_COEFFICIENTS:
            s = y.T @ y
            y = a * y + y @ (b * s + c * s @ s)
        want = 0.01 * max(g.shape) ** 0.5 * y
        assert (got.double() - want).norm() <= (0.002 + 2.0 ** -8) * want.norm() + 2.0 ** -22 * got.numel() ** 0.5
    assert torch.equal(student.shadow, student.masters.bfloat16())
