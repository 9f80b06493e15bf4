"""The example that runs the language-model operators together with the compression: it learns, raises no status bit, and
repeats bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_example_learns_and_repeats():
    from paper_2312_17530_b200 import lm_step

    losses = lm_step.run(steps=30, n_tokens=256, vocab=777, width=136, n_top=7)
    assert all(x == x and x > 0 for x in losses)
    # well over half of what can be learnt in 30 steps at this rate: the mean loss falls by a quarter at least
    assert losses[-1] < 0.75 * losses[0]
    assert lm_step.run(steps=30, n_tokens=256, vocab=777, width=136, n_top=7) == losses


def test_gradients_in_the_arena_are_the_operators_and_are_compressed():
    """A step's arena holds the three gradients between the plan's paddings, and sent + kept equals what was computed."""
    from paper_2312_17530_b200 import lm_step

    teacher = torch.randn(500, 64, device="cuda") * 0.4
    student = lm_step.Student(500, 64, 1)
    worker = lm_step.Worker(student, 96, 5, teacher, 2)
    worker.arena.fill_(7.0)
    worker.gradients(2.0)
    inside = torch.zeros_like(worker.arena, dtype=torch.bool)
    for l in student.plan.layers:
        inside[l.elem_offset:l.elem_offset + l.rows * l.cols] = True
    assert (worker.arena[~inside] == 7.0).all() and torch.isfinite(worker.arena).all()
    plan = student.plan
    resid = torch.zeros(plan.info.arena_elems, device="cuda")
    ratios = torch.full((3,), 0.1, device="cuda")
    ni, nv = plan.payload_bound(0.1)
    idx, val = torch.empty(ni, dtype=torch.int32, device="cuda"), torch.empty(nv, device="cuda")
    counts = torch.empty(3, dtype=torch.int32, device="cuda")
    ws = torch.empty(plan.info.workspace_bytes, dtype=torch.uint8, device="cuda")
    plan.compress(worker.arena, resid, ratios, idx, val, counts, workspace=ws)
    dense = torch.zeros_like(resid)
    plan.decompress_assign([(idx, val, counts)], dense)
    assert torch.equal((dense + resid)[inside], worker.arena.float()[inside])
    assert plan.status().flags == 0
