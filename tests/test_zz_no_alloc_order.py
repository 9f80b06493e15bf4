"""rsdgc_update_ratios_noalloc() without a plan, after the language-model operators: they load many kernels, and the room that the
driver had set aside for code may be full when this one's are asked for.  Each order in a process of its own, which has loaded
nothing before."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

SCRIPT = """
import sys
import torch
from paper_2312_17530_b200 import binding

def norms(kind, n, d, pad):
    x, dy = (torch.randn(n, d + pad, device="cuda").to(kind)[:, :d] for _ in range(2))
    for param in {kind, torch.float32}:
        w, m = torch.ones(d, dtype=param, device="cuda"), torch.zeros(n, device="cuda")
        y, ws = torch.empty_like(x), torch.empty(binding.layer_norm_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
        binding.layer_norm_forward(x, w, w, y, m, m.clone())
        for grad in (torch.float32, torch.bfloat16, torch.float16):
            g = torch.empty(d, dtype=grad, device="cuda")
            binding.layer_norm_backward(dy, x, w, m, m + 1, y, g, g.clone(), ws)

def heads(kind, n, v, d, k):
    H, W = (torch.randn(r, d, device="cuda").to(kind) for r in (n, v))
    f = [torch.zeros(n, device="cuda") for _ in range(3)]
    ws = torch.empty(binding.head_workspace_bytes(n, v, d, k), dtype=torch.uint8, device="cuda")
    labels, top = torch.zeros(n, dtype=torch.int64, device="cuda"), torch.zeros(n, k, dtype=torch.int64, device="cuda")
    binding.head_loss_forward(H, W, labels, f[0], f[1], ws)
    binding.head_loss_backward(H, W, labels, f[1], f[2], H.clone(), W.clone(), ws)
    for logit in (torch.float32, torch.bfloat16, torch.float16):
        q = torch.zeros(n, k, dtype=logit, device="cuda")
        binding.head_distill_forward(H, W, top, q, 1.0, f[0], f[1], ws)
        binding.head_distill_backward(H, W, top, q, 1.0, f[1], f[2], H.clone(), W.clone(), ws)

calls = []
for kind in (torch.float32, torch.bfloat16, torch.float16):
    for d, pad in ((64, 0), (64, 3), (1000, 0), (1000, 3), (4100, 0), (4100, 3), (20000, 0), (20000, 3)):
        calls.append((norms, kind, 20, d, pad))
for kind in (torch.bfloat16, torch.float16):
    calls.append((heads, kind, 20, 300, 64, 4))
w, out = torch.randn(1 << 16, device="cuda"), torch.empty(1, device="cuda")
torch.cuda.synchronize()
worst = 0
for fn, *args in calls[: int(sys.argv[1])]:
    fn(*args)
torch.cuda.synchronize()
before = torch.cuda.mem_get_info()[0]
binding.update_ratios_noalloc(w, [0], [1 << 16], 0.1, out)
torch.cuda.synchronize()
print("taken", before - torch.cuda.mem_get_info()[0])
"""


@pytest.mark.parametrize("calls", [0, 4, 26])
def test_nothing_is_allocated_after_operators(calls):
    """After the first `calls` of the list, none among them."""
    out = subprocess.run([sys.executable, "-c", SCRIPT, str(calls)], capture_output=True, text=True, timeout=300,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert out.returncode == 0, out.stderr[-2000:]
    assert out.stdout.split() == ["taken", "0"]
