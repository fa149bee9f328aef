"""The head operators -- the LM head's losses with their gradients, and the gradient of the exit projection -- and the
calls they are measured on.

    loss          softmax cross entropy of rows under an LM head, forward: a score for every token
    loss_step     the same and its gradients to the rows and the head's weights
    distill       divergence from a teacher's few largest logits, forward
    distill_step  the same and its gradients
    project_grad  gradient of the exit projection: to the row each token exited with and to the final norm's gain

`run` computes them in elementary torch operations, or with the framework's kernels where `own` is true.  Hidden sizes
are those of the repository's sweep (one of them, 1600, no multiple of 128), the sizes of the vocabulary generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
SIZES = (768, 1024, 1600, 2048, 2560, 4096, 5120, 8192)
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
# upstream gradients are divided by the number of rows; a program that runs in fp16 scales its loss up against underflow
LOSS_SCALE = {"f32": 1.0, "f16": 4096.0, "bf16": 1.0}


def _head(name, op, dtype, T, d, V, K=0, tau=1.0):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "d": d, "V": V, "K": K, "tau": tau}


def _project(name, dtype, C, T, d):
    return {"name": name, "op": "project_grad", "dtype": dtype, "C": C, "T": T, "d": d}


def listed():
    return [
        # the log-probability of one generated token at its exit, 8B model: one pass over the head's weights
        _head("loss_bf16_T1", "loss", "bf16", 1, 4096, 128000),
        # scoring the tokens of a running batch on a small model, odd vocabulary
        _head("loss_f16_T48", "loss", "f16", 48, 2048, 49157),
        # perplexity of a batch of texts at one checkpoint's exit, 8B model
        _head("loss_bf16_T4096", "loss", "bf16", 4096, 4096, 128000),
        # tuning the head on the paper's 322 prompt tokens
        _head("loss_step_bf16_T322", "loss_step", "bf16", 322, 4096, 128000),
        # a training step's micro-batch, 8B model: the largest call
        _head("loss_step_bf16_T8192", "loss_step", "bf16", 8192, 4096, 128000),
        # a model that runs in fp16, ragged batch and odd vocabulary
        _head("loss_step_f16_T2047", "loss_step", "f16", 2047, 2560, 50261),
        # a small model that runs in fp32, ragged batch
        _head("loss_step_f32_T1001", "loss_step", "f32", 1001, 1024, 32003),
        # how far a few generated tokens' exits are from the full depth's answers, fp32
        _head("distill_f32_T17", "distill", "f32", 17, 768, 32003, K=8, tau=2.0),
        # making a checkpoint's exit answer like the full depth: 2048 tokens, 32 teacher logits each
        _head("distill_step_bf16_T2048", "distill_step", "bf16", 2048, 4096, 128000, K=32, tau=2.0),
        # one token's exit row
        _project("project_grad_bf16_T1", "bf16", 8, 1, 4096),
        # the rows of a batch of prompts, hidden size that is no multiple of 128
        _project("project_grad_f32_T1361", "f32", 10, 1361, 1600),
        # the rows of the largest training step
        _project("project_grad_bf16_T8192", "bf16", 8, 8192, 4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("loss", "loss", "loss_step", "loss_step", "distill", "distill_step", "distill_step", "project_grad"))
    dtype, d = rng.choice(("bf16", "bf16", "f16", "f32")), rng.choice(SIZES)
    if op == "project_grad":
        c = {"op": op, "dtype": dtype, "C": rng.randint(4, 10), "T": _log_int(rng, 1, 16384), "d": d}
        while c["T"] * d > 8192 * 4096:
            c["T"] = c["T"] * 7 // 10
        return c
    c = {"op": op, "dtype": dtype, "T": _log_int(rng, 1, 8192), "d": d, "V": _log_int(rng, 1000, 128000), "K": 0, "tau": 1.0}
    if op.startswith("distill"):
        c["K"], c["tau"] = _log_int(rng, 1, 128), rng.choice((0.5, 1.0, 2.0, 4.0))
    while c["V"] * d > 128000 * 4096:                  # the weights are no larger than the largest listed ones
        c["V"] = c["V"] * 7 // 10
    while c["T"] * c["V"] * d > 4096 * 128000 * 4096:
        c["T"] = c["T"] * 7 // 10
    return c


def _generator(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + salt)
    return g


def _head_inputs(case, seed):
    """A head whose logits spread by 1.5 about zero, rows of unit mean square that point at some token by up to 12 logits
    (or at a mixture, the teacher's choices), targets that favour the lower token numbers, some rows without one."""
    T, d, V, K, dev, dtype = case["T"], case["d"], case["V"], case["K"], "cuda", TORCH[case["dtype"]]
    g = _generator(seed, 29)
    rand = lambda *s: torch.rand(s, generator=g, device=dev)
    randn = lambda *s: torch.randn(s, generator=g, device=dev)
    W = (randn(V, d) * (1.5 / math.sqrt(d))).to(dtype)
    x = randn(T, d)
    few = (rand(T) * 12) / 1.5**2
    s = {"W": W, "grad_loss": (0.5 + rand(T)) * (LOSS_SCALE[case["dtype"]] / T)}
    if K == 0:
        target = (rand(T) ** 3 * V).to(torch.int32).clamp_(max=V - 1)
        s["x"] = (x + few[:, None] * W[target.long()].float()).to(dtype)
        s["target"] = torch.where(rand(T) < 0.1, torch.full_like(target, -1), target)
        if T == 1:
            s["target"] = target
        return s
    first = rand(T) * V                                # K distinct tokens of a row: from anywhere, a fixed step apart
    step = V // K if V >= K else 1
    ids = ((first[:, None].long() + step * torch.arange(K, device=dev)[None, :]) % V).to(torch.int32)
    values, _ = (12.0 + 2.0 * randn(T, K)).sort(dim=1, descending=True)
    s["x"] = (x + few[:, None] * W[ids[:, 0].long()].float()).to(dtype)
    kept = torch.where(rand(T) < 0.2, (rand(T) * (K + 1)).long(), torch.full((T,), K, device=dev))    # some teachers kept fewer, a few none
    if T == 1:
        kept = torch.full((T,), K, device=dev)
    s["top_ids"] = torch.where(torch.arange(K, device=dev)[None, :] < kept[:, None], ids, torch.full_like(ids, -1)).contiguous()
    s["top_values"] = values.contiguous()
    return s


def _project_inputs(case, seed):
    """Hidden states with eight outlier channels, tokens that exit anywhere or not at all, a final norm's gain about one."""
    C, T, d, dev, dtype = case["C"], case["T"], case["d"], "cuda", TORCH[case["dtype"]]
    g = _generator(seed, 31)
    randn = lambda *s: torch.randn(s, generator=g, device=dev)
    scale = torch.ones(d, device=dev)
    scale[torch.randperm(d, generator=g, device=dev)[:8]] = 20.0
    hidden = torch.empty((C, T, d), dtype=dtype, device=dev)
    for c in range(C):
        hidden[c] = randn(T, d) * scale
    ids = [4 * c + 3 for c in range(C)]
    return {"hidden": hidden, "final": (randn(T, d) * scale).to(dtype), "ids": ids,
            "exit_layer": (4 * torch.randint(0, C + 1, (T,), generator=g, device=dev) + 3).to(torch.int32),
            "gain": 1.0 + 0.1 * randn(d), "grad_out": (randn(T, d) * (LOSS_SCALE[case["dtype"]] / T)).to(dtype)}


def prepare(case, seed):
    return {"case": case, **(_project_inputs if case["op"] == "project_grad" else _head_inputs)(case, seed)}


def _own(s):
    from paper_2603_21365_amd import tide_route as tr
    case, op = s["case"], s["case"]["op"]
    if op == "project_grad":
        return tr.exit_project_grad(s["hidden"], s["final"], s["exit_layer"], s["ids"], s["gain"], EPS, s["grad_out"])
    if op in ("loss", "loss_step"):
        loss, lse = tr.head_loss(s["x"], s["W"], s["target"])
        if op == "loss":
            return loss, lse
        return (loss, lse, *tr.head_loss_grad(s["x"], s["W"], s["target"], lse, s["grad_loss"]))
    loss, lse, z = tr.head_distill(s["x"], s["W"], s["top_values"], s["top_ids"], case["tau"])
    if op == "distill":
        return loss, lse, z
    return (loss, lse, z, *tr.head_distill_grad(s["x"], s["W"], s["top_values"], s["top_ids"], case["tau"], lse, s["grad_loss"]))


def _plain_project_grad(s):
    T, d = s["grad_out"].shape
    at = (s["exit_layer"].long() - 3) // 4                                     # the checkpoint of each token; one past the last: none
    rows = torch.cat((s["hidden"], s["final"][None]))[at, torch.arange(T, device=at.device)].float()
    dy = s["grad_out"].float()
    r = torch.rsqrt((rows * rows).mean(1, keepdim=True) + EPS)
    n = rows * r
    u = dy * s["gain"]
    grad = r * (u - n * (u * n).mean(1, keepdim=True))
    return grad.to(s["grad_out"].dtype), (dy * n).sum(0)


def _plain_lse(z):
    m = z.amax(1, keepdim=True)
    return (m + torch.log(torch.exp(z - m).sum(1, keepdim=True)))[:, 0]


def _plain_teacher(s, V, tau):
    """The teacher's probabilities over its own entries, zero where it has none."""
    ids = s["top_ids"].long()
    there = (ids >= 0) & (ids < V)
    t = torch.where(there, s["top_values"], torch.full_like(s["top_values"], -math.inf))
    m = t.amax(1, keepdim=True)
    e = torch.exp((t - torch.where(m == -math.inf, torch.zeros_like(m), m)) / tau)
    total = e.sum(1, keepdim=True)
    return torch.where(total > 0, e / total, torch.zeros_like(e)), torch.where(there, ids, torch.zeros_like(ids)), there


def _plain_head(s):
    case, op = s["case"], s["case"]["op"]
    V, tau, dtype = case["V"], case["tau"], s["x"].dtype
    x, W = s["x"].float(), s["W"].float()
    z = x @ W.T
    if op.startswith("loss"):
        y = s["target"].long()
        there = (y >= 0) & (y < V)
        y = torch.where(there, y, torch.zeros_like(y))
        lse = _plain_lse(z)
        loss = torch.where(there, lse - z.gather(1, y[:, None])[:, 0], torch.zeros_like(lse))
        out = (loss, lse)
        wanted, q, ids, scale, live = torch.ones_like(lse)[:, None], None, y[:, None], 1.0, there
    else:
        q, ids, there = _plain_teacher(s, V, tau)
        lse = _plain_lse(z / tau)
        own_z = torch.where(there, z.gather(1, ids), torch.zeros_like(q))
        terms = q * (torch.log(torch.where(q > 0, q, torch.ones_like(q))) - own_z / tau + lse[:, None])
        live = (q > 0).any(1)
        loss = torch.where(live, tau * tau * torch.where(q > 0, terms, torch.zeros_like(q)).sum(1), torch.zeros_like(lse))
        out = (loss, lse, own_z)
        wanted, scale = q, tau
    if not op.endswith("step"):
        return out
    g = torch.exp(z / tau - lse[:, None]).scatter_add_(1, ids, -wanted)
    g = torch.where((live & (s["grad_loss"] != 0))[:, None], g * (s["grad_loss"] * scale)[:, None], torch.zeros_like(g))
    return (*out, (g @ W).to(dtype), (g.T @ x).to(dtype))


def run(state):
    if own:
        return _own(state)
    return _plain_project_grad(state) if state["case"]["op"] == "project_grad" else _plain_head(state)


def work(case):
    T, d, e = case["T"], case["d"], BYTES[case["dtype"]]
    if case["op"] == "project_grad":                   # a row and its gradient in, a gradient out
        return {"bytes": 3 * T * d * e + 8 * d + 4 * T, "flops": 10 * T * d}
    V, K, products = case["V"], case["K"], 3 if case["op"].endswith("step") else 1
    outputs = (T + V) * d * e if products == 3 else 0
    return {"bytes": (T + V) * d * e + outputs + T * (12 + 12 * K), "flops": 2 * products * T * d * V}


def _exact_project_grad(case, seed):
    s = _project_inputs(case, seed)
    T, d, dev = case["T"], case["d"], "cuda"
    grad, gain = torch.empty((T, d), dtype=torch.float64, device=dev), torch.zeros(d, dtype=torch.float64, device=dev)
    table = {layer: c for c, layer in enumerate(s["ids"])}
    where = torch.tensor([table.get(e, -1) for e in s["exit_layer"].tolist()], device=dev)
    for c in range(-1, case["C"]):
        t = (where == c).nonzero()[:, 0]
        h = (s["final"] if c < 0 else s["hidden"][c])[t].double()
        rms = (h.pow(2).sum(1) / d + EPS).sqrt()[:, None]
        dy = s["grad_out"][t].double()
        gain += (dy * h / rms).sum(0)
        u = dy * s["gain"].double()
        grad[t] = u / rms - h * (u * h).sum(1, keepdim=True) / (d * rms.pow(3))
    return grad, gain


def exact(case, seed):
    if case["op"] == "project_grad":
        return _exact_project_grad(case, seed)
    s = _head_inputs(case, seed)
    T, d, V, K, tau, dev = case["T"], case["d"], case["V"], case["K"], case["tau"], "cuda"
    step = case["op"].endswith("step")
    f64 = dict(dtype=torch.float64, device=dev)
    W = s["W"].double()
    loss, lse, z_top = torch.zeros(T, **f64), torch.zeros(T, **f64), torch.zeros((T, K), **f64)
    dx, dW = torch.zeros((T, d) if step else 0, **f64), torch.zeros((V, d) if step else 0, **f64)
    rows = max(1, (1 << 29) // V)
    for a in range(0, T, rows):
        b = min(T, a + rows)
        x = s["x"][a:b].double()
        z = x.matmul(W.t()) / tau
        lse[a:b] = torch.logsumexp(z, dim=1)
        teacher = torch.zeros_like(z)                                          # what the row is taught, over the whole vocabulary
        if K == 0:
            y = s["target"][a:b].long()
            t = (y >= 0).nonzero()[:, 0]
            teacher[t, y[t]] = 1.0
            entropy = torch.zeros(b - a, **f64)
        else:
            v = s["top_values"][a:b].double().masked_fill(s["top_ids"][a:b] < 0, -math.inf)
            q = torch.nan_to_num(torch.softmax(v / tau, dim=1), nan=0.0)
            t, k = (s["top_ids"][a:b] >= 0).nonzero(as_tuple=True)
            at = s["top_ids"][a:b].long()[t, k]
            teacher.index_put_((t, at), q[t, k], accumulate=True)
            z_top[a + t, k] = z[t, at] * tau
            entropy = torch.special.entr(q).sum(1)
        total = teacher.sum(1)
        loss[a:b] = tau * tau * torch.where(total > 0, lse[a:b] - (teacher * z).sum(1) - entropy, torch.zeros_like(total))
        if step:
            p = torch.exp(z - lse[a:b, None]) * (total > 0).double()[:, None]
            p = (p - teacher) * (tau * s["grad_loss"][a:b].double())[:, None]
            dx[a:b] = p.matmul(W)
            dW += p.t().matmul(x)
    out = (loss, lse) if K == 0 else (loss, lse, z_top)
    return (*out, dx, dW) if step else out
