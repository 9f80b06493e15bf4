"""Timed cases of two more operators of a training step: the gated scan and the orthogonalised update.

The gated scan mixes a sequence's tokens, channel by channel, below the last layer norm; the orthogonalised update
is what an aggregated matrix gradient becomes before it is taken off the weights.  ``own`` selects between the plain
form (torch operations in binary32, rounded once at the end) and the library's kernels.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# the quintic whose five steps bring singular values from 0.01 .. 1 to about 0.7 .. 1.2
COEFFICIENTS = ((3.4445, -4.7750, 2.0315),) * 5
EPS = 1e-7


# ---------------------------------------------------------------------------------------------
# cases


def listed():
    return [
        # --- gated scan -------------------------------------------------------------------------
        # one more token for 16 texts that are being answered: nothing but latency
        dict(name="scan_one_token", op="scan", step="forward", b=16, t=1, d=4096, type="bf16", ragged=False, restarts=False,
             bias=True),
        # evaluation of a few texts of different lengths, an odd width, binary32
        dict(name="scan_forward_ragged", op="scan", step="forward", b=5, t=1501, d=1001, type="f32", ragged=True,
             restarts=False, bias=True),
        # one very long text
        dict(name="scan_forward_long", op="scan", step="forward", b=1, t=65536, d=1024, type="f16", ragged=False,
             restarts=False, bias=False),
        # a training batch's tokens, forward alone
        dict(name="scan_forward_batch", op="scan", step="forward", b=8, t=4096, d=4096, type="bf16", ragged=False,
             restarts=False, bias=True),
        # a training step on short texts packed one behind the other, an odd number of steps
        dict(name="scan_train_packed", op="scan", step="train", b=4, t=2047, d=1536, type="f16", ragged=True, restarts=True,
             bias=True),
        # a training step of a batch
        dict(name="scan_train_batch", op="scan", step="train", b=8, t=4096, d=4096, type="bf16", ragged=False,
             restarts=False, bias=True),
        # --- orthogonalised update ----------------------------------------------------------------
        # a small layer's gradient
        dict(name="update_small", op="update", b=1, m=256, n=512, type="f32", out="bf16"),
        # the same small matrix of many layers, in half precision
        dict(name="update_stack", op="update", b=24, m=256, n=1024, type="bf16", out="bf16"),
        # sizes that fit no tile, tall, a result with binary16's precision
        dict(name="update_odd_half", op="update", b=1, m=1501, n=777, type="f16", out="f16"),
        # an embedding-like gradient: far more rows than columns
        dict(name="update_tall", op="update", b=1, m=32000, n=1024, type="bf16", out="bf16"),
        # a wide model's square matrix, as the aggregation leaves it in binary32
        dict(name="update_square", op="update", b=1, m=4096, n=4096, type="f32", out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.6:
        b, d, t = _log_int(rng, 1, 64), _log_int(rng, 16, 8192), _log_int(rng, 1, 65536)
        if rng.random() < 0.6:
            d = (d + 7) // 8 * 8
        t = max(1, min(t, 8 * 4096 * 4096 // (b * d)))
        return dict(op="scan", step=rng.choice(["forward", "train"]), b=b, t=t, d=d, type=rng.choice(["bf16", "f16", "f32"]),
                    ragged=rng.random() < 0.4, restarts=rng.random() < 0.4, bias=rng.random() < 0.7)
    m, n = _log_int(rng, 16, 32000), _log_int(rng, 16, 8192)
    b = _log_int(rng, 1, 32) if m * n <= 1 << 20 else 1
    while b * min(m, n) * m * n > 4096 ** 3:
        m, n = (max(16, m // 2), n) if m > n else (m, max(16, n // 2))
    return dict(op="update", b=b, m=m, n=n, type=rng.choice(["bf16", "f16", "f32"]), out=rng.choice(["bf16", "bf16", "f16"]))


# ---------------------------------------------------------------------------------------------
# inputs


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = DTYPES[case["type"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    if case["op"] == "update":
        b, m, n = case["b"], case["m"], case["n"]
        # an aggregated gradient: a few directions that all tokens share, and each token's own
        r = max(1, min(m, n, 64) // 4)
        x = 0.3 * normal(b, m, n)
        x += (normal(b, m, r) / math.sqrt(r)) @ normal(b, r, n)
        x *= 1e-3
        return dict(case=case, x=x.to(dtype), out=torch.empty(b, m, n, dtype=DTYPES[case["out"]], device="cuda"))
    b, t, d = case["b"], case["t"], case["d"]
    # decays from a few tokens to some hundreds, by channel; inputs are gate logits of unit size around them
    level = 0.5 + 5.0 * uniform(d)
    s = dict(case=case, x=normal(b, t, d).to(dtype), first=normal(b, d))
    s["gate"] = normal(b, t, d)
    if case["bias"]:
        s["bias"] = level.to(dtype)
    else:
        s["bias"] = None
        s["gate"] += level
    s["gate"] = s["gate"].to(dtype)
    s["lengths"] = s["restart"] = None
    if case["ragged"]:
        s["lengths"] = (t * (0.2 + 0.8 * uniform(b))).long().clamp(max=t)
    if case["restarts"]:
        s["restart"] = uniform(b, t) < 1 / 200
    s["y"] = torch.zeros(b, t, d, dtype=dtype, device="cuda")
    s["last"] = torch.empty(b, d, device="cuda")
    if case["step"] == "train":
        s["dy"] = (normal(b, t, d) * 0.1).to(dtype)
        s["dlast"] = 0.1 * normal(b, d)
        s["dx"], s["dgate"] = torch.zeros_like(s["y"]), torch.zeros_like(s["y"])
        s["dfirst"] = torch.empty(b, d, device="cuda")
        s["dbias"] = torch.empty(d, device="cuda") if case["bias"] else None
    return s


# ---------------------------------------------------------------------------------------------
# the plain forms: binary32, rounded once at the end


def _scan(decay, add):
    """h[t] = decay[t] h[t-1] + add[t] along dimension 1, by doubling the stride."""
    stride = 1
    while stride < add.shape[1]:
        add = torch.cat([add[:, :stride], torch.addcmul(add[:, stride:], decay[:, stride:], add[:, :-stride])], 1)
        decay = torch.cat([decay[:, :stride], decay[:, stride:] * decay[:, :-stride]], 1)
        stride *= 2
    return add


def _scan_plain(s):
    x, case = s["x"].float(), s["case"]
    z = s["gate"].float()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    keep, take = torch.sigmoid(z), torch.sigmoid(-z)
    # what carries the state on: nothing where a text starts; behind a text's end the state stays
    carry, add = keep, take * x
    if s["restart"] is not None:
        carry = carry.masked_fill(s["restart"][:, :, None], 0.0)
    valid = None
    if s["lengths"] is not None:
        valid = (torch.arange(case["t"], device="cuda") < s["lengths"][:, None])[:, :, None]
        carry, add = torch.where(valid, carry, 1.0), torch.where(valid, add, 0.0)
    add = torch.cat([s["first"][:, None], add], 1)
    h = _scan(torch.cat([torch.ones_like(carry[:, :1]), carry], 1), add)
    y = h[:, 1:] if valid is None else torch.where(valid, h[:, 1:], 0.0)
    out = {"y": y.to(s["x"].dtype), "last": h[:, -1].clone()}
    if case["step"] == "train":
        dy = s["dy"].float()
        if valid is not None:
            dy = torch.where(valid, dy, 0.0)
        # from the end: delta[t] = dy[t] + carry[t+1] delta[t+1]; the last state's gradient comes first
        after = torch.cat([s["dlast"][:, None], dy.flip(1)], 1)
        back = torch.cat([torch.ones_like(carry[:, :2]), carry[:, 1:].flip(1)], 1)
        delta = _scan(back, after)[:, 1:].flip(1)
        before = h[:, :-1]
        if s["restart"] is not None:
            before = before.masked_fill(s["restart"][:, :, None], 0.0)
        dx, dz = take * delta, delta * keep * take * (before - x)
        if valid is not None:
            dx, dz = torch.where(valid, dx, 0.0), torch.where(valid, dz, 0.0)
        out |= {"dx": dx.to(s["x"].dtype), "dgate": dz.to(s["x"].dtype), "dfirst": carry[:, 0] * delta[:, 0]}
        if s["bias"] is not None:
            out["dbias"] = dz.sum((0, 1))
    return out


def _update_plain(s):
    y = s["x"].float()
    tall = y.shape[1] > y.shape[2]
    if tall:
        y = y.mT
    y = y / (y.double().square().sum((1, 2), keepdim=True).sqrt() + EPS).float()
    for a, b, c in COEFFICIENTS:
        gram = y @ y.mT
        y = a * y + (b * gram + c * (gram @ gram)) @ y
    return {"out": (y.mT if tall else y).to(s["out"].dtype)}


# ---------------------------------------------------------------------------------------------
# the library's calls


def _own(s):
    from paper_2312_17530_b200 import binding

    case = s["case"]
    if case["op"] == "update":
        if "workspace" not in s:
            size = binding.orthogonalize_workspace_bytes(case["b"], case["m"], case["n"], s["out"].dtype)
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        binding.orthogonalize(s["x"], s["out"], s["workspace"], COEFFICIENTS, EPS)
        return {"out": s["out"]}
    train = case["step"] == "train"
    if train and "states" not in s:
        s["states"] = torch.empty(binding.gated_scan_states_shape(case["b"], case["t"], case["d"]), device="cuda")
        size = binding.gated_scan_workspace_bytes(case["b"], case["t"], case["d"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    binding.gated_scan_forward(s["x"], s["gate"], s["y"], s["bias"], s["first"], s["last"], s["restart"], s["lengths"],
                               s["states"] if train else None)
    out = {"y": s["y"], "last": s["last"]}
    if train:
        binding.gated_scan_backward(s["dy"], s["x"], s["gate"], s["states"], s["dx"], s["dgate"], s["bias"], s["dbias"],
                                    s["dlast"], s["dfirst"], s["restart"], s["lengths"], s["workspace"])
        out |= {"dx": s["dx"], "dgate": s["dgate"], "dfirst": s["dfirst"]}
        if s["dbias"] is not None:
            out["dbias"] = s["dbias"]
    return out


def run(state):
    if own:
        return _own(state)
    return _update_plain(state) if state["case"]["op"] == "update" else _scan_plain(state)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "update":
        short, wide = sorted((case["m"], case["n"]))
        # the two symmetric products need half of their entries
        step = short * short * wide + short ** 3 + 2 * short * short * wide
        return {"bytes": case["b"] * case["m"] * case["n"] * (size + 2), "flops": case["b"] * len(COEFFICIENTS) * step}
    b, t, d = case["b"], case["t"], case["d"]
    n = b * t * d
    small = 8 * b * d + (size * d if case["bias"] else 0) + (8 * b if case["ragged"] else 0) + (b * t if case["restarts"] else 0)
    if case["step"] == "forward":
        return {"bytes": 3 * n * size + small, "flops": 8 * n}
    return {"bytes": 8 * n * size + 2 * small + 8 * b * d + (4 * d if case["bias"] else 0), "flops": 24 * n}


# ---------------------------------------------------------------------------------------------
# the definitions in binary64


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "update":
        x = s["x"].double()
        q = x / (torch.linalg.matrix_norm(x)[:, None, None] + EPS)
        for a, b, c in COEFFICIENTS:
            # the same polynomial from whichever side is shorter
            if case["m"] <= case["n"]:
                g = torch.einsum("bik,bjk->bij", q, q)
                q = a * q + torch.einsum("bij,bjk->bik", b * g + c * torch.matmul(g, g), q)
            else:
                g = torch.einsum("bki,bkj->bij", q, q)
                q = a * q + torch.einsum("bki,bij->bkj", q, b * g + c * torch.matmul(g, g))
        return {"out": q}
    b, t, d = case["b"], case["t"], case["d"]
    x, z = s["x"].double(), s["gate"].double()
    if s["bias"] is not None:
        z = z + s["bias"].double()
    length = s["lengths"] if s["lengths"] is not None else torch.full((b,), t, device="cuda")
    valid = torch.arange(t, device="cuda") < length[:, None]
    start = s["restart"] if s["restart"] is not None else torch.zeros_like(valid)
    h = s["first"].double()
    y = torch.zeros_like(x)
    before = torch.zeros_like(x)
    for i in range(t):
        prev = torch.where(start[:, i, None], 0.0, h)
        a = 1 / (1 + torch.exp(-z[:, i]))
        v = valid[:, i, None]
        new = a * prev + (1 - a) * x[:, i]
        before[:, i] = prev
        h = torch.where(v, new, h)
        y[:, i] = torch.where(v, new, 0.0)
    out = {"y": y, "last": h}
    if case["step"] == "train":
        dx, dz = torch.zeros_like(x), torch.zeros_like(x)
        g = s["dlast"].double()  # of the state behind the step
        for i in reversed(range(t)):
            v = valid[:, i, None]
            a = 1 / (1 + torch.exp(-z[:, i]))
            e = g + s["dy"][:, i].double()
            dx[:, i] = torch.where(v, (1 - a) * e, 0.0)
            dz[:, i] = torch.where(v, e * (before[:, i] - x[:, i]) * a * (1 - a), 0.0)
            g = torch.where(v, torch.where(start[:, i, None], 0.0, a * e), g)
        out |= {"dx": dx, "dgate": dz, "dfirst": g}
        if s["bias"] is not None:
            out["dbias"] = dz.sum((0, 1))
    return out
