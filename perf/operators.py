"""Timed cases of the language-model operators: layer norm, the vocabulary head's loss, distillation.

These three are the end of a language model's training step: the last layer norm, the product with
the vocabulary matrix with its softmax cross entropy, and the same head trained towards a teacher's
top logits.  Their weight gradients are what the compression step takes in.  ``own`` selects between
the plain form (torch operations in binary32, rounded once at the end) and the library's kernels.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------------------------
# cases


def listed():
    return [
        # --- layer norm -------------------------------------------------------------------------
        # one token of a model that is answering: nothing but latency
        dict(name="norm_forward_one_token", op="norm", step="forward", n=1, d=4096, type="bf16", params="bf16"),
        # an odd width, binary32: no row but the first starts on a 16-byte boundary
        dict(name="norm_forward_odd_width", op="norm", step="forward", n=1500, d=1001, type="f32", params="f32"),
        # a training batch's tokens through one norm
        dict(name="norm_forward_batch", op="norm", step="forward", n=16384, d=4096, type="bf16", params="bf16"),
        # a small model's batch in half precision with binary32 parameters
        dict(name="norm_backward_half", op="norm", step="backward", n=2048, d=1000, type="f16", params="f32"),
        # a wide model's batch: the weight's gradient sums 16384 rows
        dict(name="norm_backward_batch", op="norm", step="backward", n=16384, d=8192, type="bf16", params="bf16"),
        # --- cross entropy over the vocabulary ---------------------------------------------------
        # scoring the end of one short answer with a small head
        dict(name="loss_forward_few_tokens", op="loss", step="forward", n=5, v=1000, d=256, type="bf16", ignored=0.0),
        # evaluation: the loss of a batch, no gradient
        dict(name="loss_forward_batch", op="loss", step="forward", n=2048, v=32000, d=2048, type="f16", ignored=0.0),
        # a training step whose tokens, vocabulary and width fit no tile, with padding tokens
        dict(name="loss_step_ragged", op="loss", step="train", n=1023, v=50001, d=1000, type="bf16", ignored=0.1),
        # a training step of a large head
        dict(name="loss_step_large", op="loss", step="train", n=8192, v=128000, d=4096, type="bf16", ignored=0.02),
        # --- distillation from a teacher's top logits -------------------------------------------
        # how far a student is from its teacher, on a short text; some tokens have fewer entries
        dict(name="distill_forward_ragged", op="distill", step="forward", n=333, v=10007, d=776, k=20, type="f16",
             ignored=0.1),
        # a training step of a tiny student
        dict(name="distill_step_small", op="distill", step="train", n=64, v=8000, d=512, k=8, type="f16", ignored=0.0),
        # a training step of an ordinary student
        dict(name="distill_step_batch", op="distill", step="train", n=2048, v=32000, d=2048, k=64, type="bf16",
             ignored=0.05),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "loss", "distill"])
    kind = rng.choice(["bf16", "f16"])
    if op == "norm":
        n, d = _log_int(rng, 1, 16384), _log_int(rng, 64, 16384)
        n = max(1, min(n, 16384 * 8192 // d))
        kind = rng.choice(["bf16", "f16", "f32"])
        return dict(op="norm", step=rng.choice(["forward", "backward"]), n=n, d=d, type=kind,
                    params=rng.choice([kind, "f32"]))
    n, v, d = _log_int(rng, 1, 8192), _log_int(rng, 500, 128000), _log_int(rng, 64, 4096)
    if rng.random() < 0.7:
        d = (d + 7) // 8 * 8
    case = dict(op=op, step=rng.choice(["forward", "train"]), n=n, v=v, d=d, type=kind,
                ignored=rng.choice([0.0, 0.05, 0.3]))
    if op == "distill":
        case["k"] = _log_int(rng, 1, 128)
    return case


# ---------------------------------------------------------------------------------------------
# inputs


def _rows(gen, n, d, dtype):
    """n x d normal values whose rows start on 16-byte boundaries, as a padded buffer keeps them."""
    pitch = (d + 7) // 8 * 8
    buf = torch.zeros(n, pitch, dtype=dtype, device="cuda")
    buf[:, :d] = torch.randn(n, d, generator=gen, device="cuda").to(dtype)
    return buf[:, :d]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, d, dtype = case["n"], case["d"], DTYPES[case["type"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    if case["op"] == "norm":
        params = DTYPES[case["params"]]
        # a residual stream: every token has its own scale and offset, some channels are far larger
        x = normal(n, d) * (0.5 + 2 * uniform(n, 1)) + 0.3 * normal(n, 1) + 0.2
        x *= torch.where(uniform(d) < 0.01, 8.0, 1.0)
        x = x.to(dtype)
        s = dict(case=case, x=x, w=(1 + 0.2 * normal(d)).to(params), b=(0.1 * normal(d)).to(params), eps=1e-5,
                 mean=torch.empty(n, device="cuda"), rstd=torch.empty(n, device="cuda"))
        if case["step"] == "forward":
            s["y"] = torch.empty_like(x)
        else:
            f = x.float()
            s["mean"] = f.mean(1)
            s["rstd"] = torch.rsqrt((f - s["mean"][:, None]).square().mean(1) + s["eps"])
            s["dy"] = (normal(n, d) * 0.1).to(dtype)
            s["dx"] = torch.empty_like(x)
            s["dw"] = torch.empty(d, dtype=params, device="cuda")
            s["db"] = torch.empty(d, dtype=params, device="cuda")
        return s

    v = case["v"]
    weight = _rows(gen, v, d, dtype)
    weight.mul_(2.0 / math.sqrt(d))  # logits of a few units
    none = uniform(n) < case["ignored"]
    s = dict(case=case, weight=weight, loss=torch.empty(n, device="cuda"), lse=torch.empty(n, device="cuda"))
    if case["op"] == "loss":
        labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
        best = labels
        s["labels"] = torch.where(none, -1, labels)
    else:
        k = case["k"]
        # k different entries of the vocabulary per token, best first; some tokens have fewer, some none
        gaps = torch.randint(1, max(2, v // k), (n, k), generator=gen, device="cuda")
        index = (torch.randint(0, v, (n, 1), generator=gen, device="cuda") + gaps.cumsum(1)) % v
        index = index.gather(1, uniform(n, k).argsort(1))
        s["top_logit"] = (2.5 * normal(n, k)).sort(1, descending=True).values.contiguous()
        best = index[:, 0]
        fewer = (uniform(n, 1) < 0.2) & (torch.arange(k, device="cuda") >= (k + 1) // 2)
        s["top_index"] = torch.where(none[:, None] | fewer, -1, index).contiguous()
        s["temperature"] = 2.0
    # a student that has learnt something: its best guess leans towards the wanted entry
    hidden = _rows(gen, n, d, dtype)
    hidden.copy_((hidden.float() + weight[best].float()).to(dtype))
    s["hidden"] = hidden
    if case["step"] == "train":
        scale = 1024.0 if case["type"] == "f16" else 1.0  # half-precision training scales its loss
        s["grad"] = scale * (0.5 + uniform(n)) / n
        s["dhidden"] = torch.empty(n, d, dtype=dtype, device="cuda")
        s["dweight"] = torch.empty(v, d, dtype=dtype, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------
# the plain forms: binary32, rounded once at the end


def _norm_forward(s):
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = torch.rsqrt(c.square().mean(1) + s["eps"])
    y = c * rstd[:, None] * w + b
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _norm_backward(s):
    x, w, dy = s["x"].float(), s["w"].float(), s["dy"].float()
    xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * w
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dw": (dy * xhat).sum(0).to(s["w"].dtype), "db": dy.sum(0).to(s["w"].dtype)}


def _softmax_parts(z):
    m = z.max(1, keepdim=True).values
    e = (z - m).exp_()
    t = e.sum(1, keepdim=True)
    return e, t, (m + t.log()).squeeze(1)


def _head_gradients(s, hidden, weight, dz):
    return {"dhidden": (dz @ weight).to(s["hidden"].dtype), "dweight": (dz.T @ hidden).to(s["weight"].dtype)}


def _loss(s):
    hidden, weight, labels = s["hidden"].float(), s["weight"].float(), s["labels"]
    z = hidden @ weight.T
    e, t, lse = _softmax_parts(z)
    valid = labels >= 0
    at = labels.clamp(min=0)[:, None]
    loss = torch.where(valid, lse - z.gather(1, at).squeeze(1), 0.0)
    out = {"loss": loss, "lse": lse}
    if s["case"]["step"] == "train":
        g = torch.where(valid, s["grad"], 0.0)[:, None]
        dz = e.mul_(g / t).scatter_add_(1, at, -g)
        out |= _head_gradients(s, hidden, weight, dz)
    return out


def _distill(s):
    hidden, weight, index, T = s["hidden"].float(), s["weight"].float(), s["top_index"], s["temperature"]
    z = (hidden @ weight.T).mul_(1.0 / T)
    e, t, lse = _softmax_parts(z)
    valid = index >= 0
    some = valid.any(1)
    at = index.clamp(min=0)
    u = torch.where(valid, s["top_logit"] / T, -math.inf)
    u = torch.where(some[:, None], u - u.max(1, keepdim=True).values, 0.0)
    q = torch.where(valid, u.exp(), 0.0)
    total = q.sum(1, keepdim=True).clamp(min=1e-30)
    q = q / total
    log_q = torch.where(valid, u - total.log(), 0.0)
    loss = T * T * (q * torch.where(valid, log_q - (z.gather(1, at) - lse[:, None]), 0.0)).sum(1)
    out = {"loss": loss, "lse": lse}
    if s["case"]["step"] == "train":
        g = torch.where(some, s["grad"] * T, 0.0)[:, None]
        dz = e.mul_(g / t).scatter_add_(1, at, -g * q)
        out |= _head_gradients(s, hidden, weight, dz)
    return out


# ---------------------------------------------------------------------------------------------
# the library's calls


def _own(s):
    from paper_2312_17530_b200 import binding

    case = s["case"]
    if case["op"] == "norm":
        if case["step"] == "forward":
            binding.layer_norm_forward(s["x"], s["w"], s["b"], s["y"], s["mean"], s["rstd"], s["eps"])
            return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        if "workspace" not in s:
            size = binding.layer_norm_workspace_bytes(case["n"], case["d"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        binding.layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"],
                                    s["workspace"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if "workspace" not in s:
        size = binding.head_workspace_bytes(case["n"], case["v"], case["d"], case.get("k", 1))
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    if case["op"] == "loss":
        binding.head_loss_forward(s["hidden"], s["weight"], s["labels"], s["loss"], s["lse"], s["workspace"])
    else:
        binding.head_distill_forward(s["hidden"], s["weight"], s["top_index"], s["top_logit"], s["temperature"],
                                     s["loss"], s["lse"], s["workspace"])
    out = {"loss": s["loss"], "lse": s["lse"]}
    if case["step"] == "train":
        if case["op"] == "loss":
            binding.head_loss_backward(s["hidden"], s["weight"], s["labels"], s["lse"], s["grad"], s["dhidden"],
                                       s["dweight"], s["workspace"])
        else:
            binding.head_distill_backward(s["hidden"], s["weight"], s["top_index"], s["top_logit"],
                                          s["temperature"], s["lse"], s["grad"], s["dhidden"], s["dweight"],
                                          s["workspace"])
        out |= {"dhidden": s["dhidden"], "dweight": s["dweight"]}
    return out


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["op"] == "norm":
        return _norm_forward(state) if case["step"] == "forward" else _norm_backward(state)
    return _loss(state) if case["op"] == "loss" else _distill(state)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    n, d = case["n"], case["d"]
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "norm":
        par = 4 if case["params"] == "f32" else 2
        if case["step"] == "forward":
            return {"bytes": 2 * n * d * size + 2 * d * par + 8 * n, "flops": 8 * n * d}
        return {"bytes": 3 * n * d * size + 3 * d * par + 8 * n, "flops": 14 * n * d}
    v, k = case["v"], case.get("k", 0)
    moved = (n * d + v * d) * size + 16 * n + 12 * n * k
    if case["step"] == "forward":
        return {"bytes": moved, "flops": 2 * n * v * d}
    # the logits' product and the two products of the gradients
    return {"bytes": moved + (n * d + v * d) * size + 4 * n, "flops": 6 * n * v * d}


# ---------------------------------------------------------------------------------------------
# the definitions in binary64


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x, w = s["x"].double(), s["w"].double()
        d = case["d"]
        if case["step"] == "forward":
            mean = x.sum(1) / d
            var = ((x - mean.unsqueeze(1)) ** 2).sum(1) / d
            rstd = 1 / torch.sqrt(var + s["eps"])
            return {"y": torch.addcmul(s["b"].double(), (x - mean.unsqueeze(1)) / torch.sqrt(var + s["eps"]).unsqueeze(1), w),
                    "mean": mean, "rstd": rstd}
        dy, rstd = s["dy"].double(), s["rstd"].double().unsqueeze(1)
        xhat = (x - s["mean"].double().unsqueeze(1)) * rstd
        # y = w * xhat + b, xhat = (x - mean) * rstd: the two statistics depend on every x of the row
        along = (dy * w * xhat).sum(1, keepdim=True) / d
        across = (dy * w).sum(1, keepdim=True) / d
        return {"dx": rstd * (dy * w - across - xhat * along), "dw": torch.einsum("nd,nd->d", dy, xhat),
                "db": torch.einsum("nd->d", dy)}
    n, v, d = case["n"], case["v"], case["d"]
    T = s.get("temperature", 1.0)
    W = s["weight"].double()
    loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(loss)
    train = case["step"] == "train"
    if train:
        dh = torch.zeros(n, d, dtype=torch.float64, device="cuda")
        dw = torch.zeros(v, d, dtype=torch.float64, device="cuda")
    for r in range(0, n, 1024):
        rows = slice(r, min(n, r + 1024))
        H = s["hidden"][rows].double()
        logp = torch.log_softmax(H @ W.T / T, 1)
        lse[rows] = (H @ W[0]) / T - logp[:, 0]
        target = torch.zeros_like(logp)  # the wanted distribution, dense
        if case["op"] == "loss":
            lab = s["labels"][rows]
            here = torch.nonzero(lab >= 0).squeeze(1)
            target[here, lab[here]] = 1.0
            loss[rows] = -(target * logp).sum(1)
        else:
            idx, top = s["top_index"][rows], s["top_logit"][rows].double() / T
            q = torch.nan_to_num(torch.softmax(top.masked_fill(idx < 0, -math.inf), 1), nan=0.0)
            target.scatter_add_(1, idx.clamp(min=0), q)
            own_part = torch.where(q > 0, q * torch.log(q.clamp(min=1e-300)), 0.0).sum(1)
            loss[rows] = T * T * (own_part - (target * logp).sum(1))
        if train:
            # d loss / d z of the unscaled logits; a row with no target has no loss
            mass = target.sum(1, keepdim=True)
            dz = (logp.exp_() * mass - target) * (s["grad"][rows].double() * (T if case["op"] == "distill" else 1.0)).unsqueeze(1)
            dh[rows] = dz @ W
            dw += dz.T @ H
    out = {"loss": loss, "lse": lse}
    if train:
        out |= {"dhidden": dh, "dweight": dw}
    return out
