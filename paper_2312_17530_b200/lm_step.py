"""A language model's last layers trained with compressed gradients, as a small runnable example.

Several workers share one GPU.  Each normalises its tokens' activations (layer norm), then trains the
vocabulary head: half of its tokens towards labels (cross entropy), half towards a teacher's top logits
(distillation).  The gradients of the head's matrix and of the norm's parameters are written straight
into the worker's gradient arena, the workers' arenas are compressed in one call, the payloads are
aggregated into a dense gradient, and the masters take a step of SGD.  Data and teacher are synthetic.

    python -m paper_2312_17530_b200.lm_step --steps 40
"""
from __future__ import annotations

import argparse
import json
import sys

import torch

from . import binding


class Student:
    """Binary32 masters in one arena (head, norm weight, norm bias) with the bfloat16 copies the kernels read."""

    def __init__(self, vocab: int, width: int, seed: int):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        # one layer per parameter: the head in 3 x 3 neighborhoods, the vectors in runs of 9
        self.plan = binding.Plan([(vocab, width, 3, 3), (1, width, 1, 9), (1, width, 1, 9)], grad_dtype=binding.RSDGC_BF16,
                                 device=torch.cuda.current_device())
        self.masters = torch.zeros(self.plan.info.arena_elems, device="cuda")
        head, weight, _ = self.views(self.masters)
        head.copy_(0.02 * torch.randn(vocab, width, generator=gen, device="cuda"))
        weight.fill_(1.0)
        self.shadow = self.masters.to(torch.bfloat16)

    def views(self, arena):
        """(head, norm weight, norm bias) inside an arena."""
        at = [arena[l.elem_offset:l.elem_offset + l.rows * l.cols] for l in self.plan.layers]
        return at[0].view(self.plan.layers[0].rows, self.plan.layers[0].cols), at[1], at[2]

    def step(self, dense, rate: float) -> None:
        self.masters.sub_(dense, alpha=rate)
        self.shadow.copy_(self.masters)


class Worker:
    """One worker's tokens and buffers; ``gradients`` fills its arena."""

    def __init__(self, student: Student, n_tokens: int, n_top: int, teacher, seed: int):
        vocab, width = teacher.shape
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.student, self.half, self.n_top = student, n_tokens // 2, n_top
        self.x = torch.randn(n_tokens, width, generator=gen, device="cuda").to(torch.bfloat16)
        logits = self.x.float() @ teacher.T
        self.labels = logits[:self.half].argmax(1)
        top = logits[self.half:].topk(n_top, dim=1)
        self.top_index, self.top_logit = top.indices.contiguous(), top.values.contiguous()
        # the padding at the end of a text has no label
        self.labels[-max(1, self.half // 16):] = -1

        def empty(*shape, dtype=torch.float32):
            return torch.empty(*shape, dtype=dtype, device="cuda")

        self.hidden, self.dhidden = torch.empty_like(self.x), torch.empty_like(self.x)
        self.mean, self.rstd = empty(n_tokens), empty(n_tokens)
        self.loss, self.lse = empty(n_tokens), empty(n_tokens)
        self.grad_loss = torch.full((n_tokens,), 1.0 / n_tokens, device="cuda")
        self.dhead = empty(vocab, width, dtype=torch.bfloat16)
        self.arena = torch.zeros(student.plan.info.arena_elems, dtype=torch.bfloat16, device="cuda")
        size = max(binding.head_workspace_bytes(n_tokens, vocab, width, n_top),
                   binding.layer_norm_workspace_bytes(n_tokens, width))
        self.workspace = empty(size, dtype=torch.uint8)

    def gradients(self, temperature: float) -> None:
        head, weight, bias = self.student.views(self.student.shadow)
        dhead, dweight, dbias = self.student.views(self.arena)
        labelled, taught, ws = slice(0, self.half), slice(self.half, None), self.workspace
        binding.layer_norm_forward(self.x, weight, bias, self.hidden, self.mean, self.rstd)
        h, dh = self.hidden[labelled], self.dhidden[labelled]
        binding.head_loss_forward(h, head, self.labels, self.loss[labelled], self.lse[labelled], ws)
        binding.head_loss_backward(h, head, self.labels, self.lse[labelled], self.grad_loss[labelled], dh, dhead, ws)
        h, dh = self.hidden[taught], self.dhidden[taught]
        binding.head_distill_forward(h, head, self.top_index, self.top_logit, temperature, self.loss[taught], self.lse[taught],
                                     ws)
        binding.head_distill_backward(h, head, self.top_index, self.top_logit, temperature, self.lse[taught],
                                      self.grad_loss[taught], dh, self.dhead, ws)
        dhead.add_(self.dhead)
        binding.layer_norm_backward(self.dhidden, self.x, weight, self.mean, self.rstd, None, dweight, dbias, ws)


def run(steps: int = 40, n_workers: int = 2, n_tokens: int = 512, vocab: int = 2000, width: int = 256, n_top: int = 16,
        ratio: float = 1 / 16, rate: float = 8.0, temperature: float = 2.0, seed: int = 0):
    """Trains and returns the mean loss per step as a list."""
    if width < 8 or width % 8:
        # the head lies in an arena's layer, whose rows have no padding, and its rows have to start on 16-byte boundaries
        raise ValueError("width: a multiple of 8 is wanted, got %d" % width)
    if n_tokens < 2 or not 1 <= n_top <= min(vocab, 1024):
        raise ValueError("two tokens or more, and 1 to min(vocab, 1024) top logits are wanted")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    teacher = torch.randn(vocab, width, generator=gen, device="cuda") * (3.0 / width ** 0.5)
    student = Student(vocab, width, seed + 1)
    plan = student.plan
    workers = [Worker(student, n_tokens, n_top, teacher, seed + 2 + w) for w in range(n_workers)]
    plan.reserve_workers(n_workers)
    ni, nv = plan.payload_bound(ratio)
    resid = [torch.zeros(plan.info.arena_elems, device="cuda") for _ in workers]
    idx = [torch.empty(ni, dtype=torch.int32, device="cuda") for _ in workers]
    val = [torch.empty(nv, device="cuda") for _ in workers]
    counts = [torch.empty(plan.n_layers, dtype=torch.int32, device="cuda") for _ in workers]
    ratios = torch.full((plan.n_layers,), ratio, device="cuda")
    workspace = torch.empty(n_workers * plan.info.workspace_bytes, dtype=torch.uint8, device="cuda")
    dense = torch.zeros(plan.info.arena_elems, device="cuda")
    losses = []
    for _ in range(steps):
        for w in workers:
            w.gradients(temperature)
        plan.compress_workers([w.arena for w in workers], resid, ratios, idx, val, counts, workspace)
        plan.decompress_assign(list(zip(idx, val, counts)), dense, 1.0 / n_workers)
        student.step(dense, rate)
        losses.append(torch.stack([w.loss.mean() for w in workers]).mean())
    status = plan.status().flags | binding.operator_status()
    if status:
        raise RuntimeError("device status %d" % status)
    return [float(x) for x in losses]


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=2000)
    ap.add_argument("--width", type=int, default=256)
    args = ap.parse_args()
    losses = run(args.steps, args.workers, args.tokens, args.vocab, args.width)
    print(json.dumps({"steps": args.steps, "loss_first": losses[0], "loss_last": losses[-1]}))
    return 0 if losses[-1] < losses[0] else 1


if __name__ == "__main__":
    sys.exit(main())
