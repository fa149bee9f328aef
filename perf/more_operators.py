"""The answer operators -- the LM head in four bits, and the rules that a decoding program puts on its logits -- and the calls
they are measured on.

    quantize  a head's weights to four bits with a scale per group of columns, and back to the values that these stand for
    logits    rows under such a head: every token's logit
    rules     penalties for repeated tokens, biases and a grammar's mask on logits
    pick      the same, but the token with the largest of them and its log-probability in their place

`run` computes them in elementary torch operations, or with the framework's kernels where `own` is true.  Hidden sizes
are those of the repository's sweep (one of them, 1600, no multiple of 128), the sizes of the vocabulary generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

SIZES = (768, 1024, 1600, 2048, 2560, 4096, 5120, 8192)
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
SCALE_BITS = {"f16": 11, "bf16": 8}


def _quantize(name, dtype, V, d, group, scale="bf16"):
    return {"name": name, "op": "quantize", "dtype": dtype, "V": V, "d": d, "group": group, "scale": scale}


def _logits(name, dtype, T, d, V, group, scale="bf16"):
    return {"name": name, "op": "logits", "dtype": dtype, "T": T, "d": d, "V": V, "group": group, "scale": scale}


def _rules(name, op, dtype, T, V, H, B, grammar=True):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "V": V, "H": H, "B": B, "grammar": grammar}


def listed():
    return [
        # one generated token at its exit, 8B model: one pass over the head's weights
        _logits("logits_bf16_T1", "bf16", 1, 4096, 128000, 128),
        # a few sequences on a small model that runs in fp16: odd vocabulary, hidden size that is no multiple of 128
        _logits("logits_f16_T5", "f16", 5, 1600, 49157, 64, "f16"),
        # a small model that runs in fp32, fine groups
        _logits("logits_f32_T3", "f32", 3, 1024, 32003, 32),
        # a running batch, 8B model
        _logits("logits_bf16_T48", "bf16", 48, 4096, 128000, 128),
        # every position of a batch of drafted or prompt tokens: the largest call
        _logits("logits_bf16_T512", "bf16", 512, 4096, 128000, 128),
        # loading a model's head: once per program, but over all of its weights
        _quantize("quantize_bf16", "bf16", 128000, 4096, 128),
        # a head that was trained in fp32, fine groups, odd vocabulary
        _quantize("quantize_f32", "f32", 32003, 1600, 32),
        # one sequence's logits before a program's own sampling
        _rules("rules_f32_T1", "rules", "f32", 1, 128000, 700, 8),
        # the logits of a batch as a model in bf16 leaves them, odd vocabulary, long biases
        _rules("rules_bf16_T64", "rules", "bf16", 64, 50261, 2049, 300),
        # one sequence's next token
        _rules("pick_f32_T1", "pick", "f32", 1, 128000, 700, 8),
        # a small batch with long pasts on a model that runs in fp16
        _rules("pick_f16_T17", "pick", "f16", 17, 49157, 30011, 0, False),
        # a large batch, 8B model
        _rules("pick_f32_T256", "pick", "f32", 256, 128000, 4096, 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("logits", "logits", "logits", "logits", "quantize", "rules", "rules", "pick", "pick"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op in ("rules", "pick"):
        dtype = rng.choice(("f32", "f32", "f16", "bf16"))
        c = {"op": op, "dtype": dtype, "T": _log_int(rng, 1, 512), "V": _log_int(rng, 1000, 200000), "H": _log_int(rng, 1, 32768),
             "B": rng.choice((0, _log_int(rng, 1, 1024))), "grammar": rng.random() < 0.7}
        while c["T"] * (c["V"] + c["H"]) > 256 * 132096:
            c["T"] = c["T"] * 7 // 10
        return c
    c = {"op": op, "dtype": dtype, "V": _log_int(rng, 1000, 200000), "d": rng.choice(SIZES), "group": rng.choice((32, 64, 128)), "scale": rng.choice(("bf16", "bf16", "f16"))}
    while c["V"] * c["d"] > 128000 * 4096:             # the weights are no larger than the largest listed ones
        c["V"] = c["V"] * 7 // 10
    if op == "logits":
        c["T"] = _log_int(rng, 1, 1024)
        while c["T"] * c["V"] * c["d"] > 512 * 128000 * 4096:
            c["T"] = c["T"] * 7 // 10
    return c


def _generator(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + salt)
    return g


def _weights(case, seed):
    """A head whose rows differ in size, and whose columns do: a few carry an outlier."""
    V, d, dev = case["V"], case["d"], "cuda"
    g = _generator(seed, 41)
    W = torch.randn((V, d), generator=g, device=dev)
    W *= (0.5 + torch.rand((V, 1), generator=g, device=dev)) * (1.5 / math.sqrt(d))
    W[:, torch.randperm(d, generator=g, device=dev)[:8]] *= 4.0
    return {"W": W.to(TORCH[case["dtype"]])}


def _lay_out(codes, scales):
    """Codes 0 .. 15 [V,d] and scales [V, groups] as the head's kernels take them: tiles of 16 rows and 128 columns, what is missing of them filled up.
    Eight columns of a row are a 32-bit word, the even ones in its lower half; a tile is 64 times four such words, 32 columns apart."""
    V, d = codes.shape
    rows, blocks = -(-V // 16), -(-d // 128)
    full = torch.full((rows * 16, blocks * 128), 8, dtype=torch.uint8, device=codes.device)
    full[:V, :d] = codes
    t = full.view(rows, 16, blocks, 4, 4, 4, 2).permute(0, 2, 4, 1, 3, 6, 5).reshape(rows, blocks, 1024, 2)
    s = torch.zeros((rows * 16, scales.shape[1]), dtype=scales.dtype, device=scales.device)
    s[:V] = scales
    return (t[..., 0] | (t[..., 1] << 4)).contiguous(), s.view(rows, 16, -1).transpose(1, 2).contiguous()


def _head(case, seed):
    """A head in four bits -- codes of rounded normal weights, scales that differ by row and group -- and rows with some outlier channels."""
    T, d, V, group, dev = case["T"], case["d"], case["V"], case["group"], "cuda"
    g = _generator(seed, 43)
    randn = lambda *s: torch.randn(s, generator=g, device=dev)
    codes = (randn(V, d) * 2.4).round_().clamp_(-7, 7).add_(8).to(torch.uint8)
    scales = ((0.5 + torch.rand((V, -(-d // group)), generator=g, device=dev)) * (0.6 / math.sqrt(d))).to(TORCH[case["scale"]])
    codes, scales = _lay_out(codes, scales)
    x = randn(T, d)
    x[:, torch.randperm(d, generator=g, device=dev)[:8]] *= 8.0
    return {"x": x.to(TORCH[case["dtype"]]), "codes": codes, "scales": scales}


def _logit_inputs(case, seed):
    """Logits with a few candidates in front of the rest, pasts of different lengths in which low token numbers are frequent, each sequence with
    penalties of its own, biases of which some ban their token, masks that leave a few tokens, everything, or (one row of a larger batch) nothing."""
    T, V, H, B, dev = case["T"], case["V"], case["H"], case["B"], "cuda"
    g = _generator(seed, 47)
    rand = lambda *s: torch.rand(s, generator=g, device=dev)
    randn = lambda *s: torch.randn(s, generator=g, device=dev)
    tokens = lambda *s: (rand(*s) ** 3 * V).to(torch.int32).clamp_(max=V - 1)
    z = randn(T, V) * 2.5 - 2.0
    z += (rand(T, V) < 16 / V) * (6.0 + 4.0 * rand(T, V))
    length = (H - (rand(T) * (H // 2)).long()).to(torch.int32)
    past = tokens(T, H)
    s = {"z": z.to(TORCH[case["dtype"]]), "past": torch.where(torch.arange(H, device=dev)[None, :] < length[:, None], past, torch.full_like(past, -1)),
         "past_len": length, "prompt_len": (length * rand(T)).to(torch.int32),
         "repetition": 1.0 + 0.5 * rand(T), "presence": rand(T) * (rand(T) < 0.7), "frequency": 0.5 * rand(T) * (rand(T) < 0.7),
         "bias_ids": None, "bias_values": None, "allowed": None}
    if B:
        values = 2.0 * randn(T, B)
        s["bias_values"] = torch.where(rand(T, B) < 0.1, torch.full_like(values, -100.0), values)
        s["bias_ids"] = torch.where(rand(T, B) < 0.1, torch.full((T, B), -1, dtype=torch.int32, device=dev), tokens(T, B))
    if case["grammar"]:
        bit = 1 << torch.arange(32, device=dev)
        few = ((rand(T, -(-V // 32), 32) < 0.02).long() * bit).sum(2)
        words = torch.where((rand(T) < 0.5)[:, None], few, torch.full_like(few, (1 << 32) - 1))
        if T >= 16:
            words[T // 2] = 0
        s["allowed"] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return s


def prepare(case, seed):
    make = {"quantize": _weights, "logits": _head}.get(case["op"], _logit_inputs)
    return {"case": case, **make(case, seed)}


def _own(s):
    from paper_2603_21365_amd import tide_route as tr
    case, op = s["case"], s["case"]["op"]
    if op == "quantize":
        codes, scales = tr.head_quantize_q4(s["W"], case["group"], scale_dtype=TORCH[case["scale"]])
        return tr.head_dequantize_q4(codes, scales, case["V"], case["d"], s["W"].dtype, case["group"])
    if op == "logits":
        return tr.head_logits_q4(s["x"], s["codes"], s["scales"], case["V"], case["group"])
    call = tr.logit_rules if op == "rules" else tr.logit_pick
    return call(s["z"], past=s["past"], past_len=s["past_len"], prompt_len=s["prompt_len"], repetition=s["repetition"], presence=s["presence"],
                frequency=s["frequency"], bias_ids=s["bias_ids"], bias_values=s["bias_values"], allowed=s["allowed"])


def _rounded(x, bits):
    """Positive normal values in 64 bits, rounded to that many significant bits, ties to even."""
    drop = 53 - bits
    word = x.view(torch.int64)
    word = word + ((1 << (drop - 1)) - 1) + ((word >> drop) & 1)
    return ((word >> drop) << drop).view(torch.float64)


def _plain_quantize(s):
    case = s["case"]
    V, d, group = case["V"], case["d"], case["group"]
    W = torch.zeros((V, -(-d // group) * group), dtype=torch.float64, device=s["W"].device)
    W[:, :d] = s["W"]
    W = W.view(V, -1, group)
    most = W.abs().amax(2, keepdim=True)
    scale = torch.where(most > 0, _rounded(most / 7, SCALE_BITS[case["scale"]]), torch.zeros_like(most))
    q = torch.round(W / torch.where(scale > 0, scale, torch.ones_like(scale)))
    return (q * scale).view(V, -1)[:, :d].to(torch.float32).to(s["W"].dtype)


def _plain_logits(s):
    case, codes = s["case"], s["codes"]
    V, d, rows, blocks = case["V"], case["d"], codes.shape[0], codes.shape[1]
    q = torch.stack((codes & 15, codes >> 4), 3).view(rows, blocks, 4, 16, 4, 2, 4).permute(0, 3, 1, 4, 2, 6, 5).reshape(rows * 16, blocks * 128)[:V, :d]
    scale = s["scales"].float().transpose(1, 2).reshape(rows * 16, -1)[:V].repeat_interleave(case["group"], dim=1)[:, :d]
    return s["x"].float() @ ((q.float() - 8.0) * scale).T


def _plain_ruled(s):
    z, past = s["z"].float(), s["past"].long()
    T, V = z.shape
    at = torch.arange(past.shape[1], device=z.device)[None, :]
    there = (past >= 0) & (past < V) & (at < s["past_len"][:, None])
    own_part = there & (at >= s["prompt_len"][:, None])
    token = torch.where(there, past, torch.zeros_like(past))
    seen = torch.zeros_like(z).scatter_add_(1, token, there.float())
    count = torch.zeros_like(z).scatter_add_(1, token, own_part.float())
    rho = s["repetition"][:, None]
    z = torch.where(seen > 0, torch.where(z > 0, z / rho, z * rho), z)
    z = torch.where(count > 0, z - (s["frequency"][:, None] * count + s["presence"][:, None]), z)
    if s["bias_ids"] is not None:
        ids = s["bias_ids"].long()
        there = (ids >= 0) & (ids < V)
        z = z + torch.zeros_like(z).scatter_add_(1, torch.where(there, ids, torch.zeros_like(ids)), torch.where(there, s["bias_values"], torch.zeros_like(s["bias_values"])))
    if s["allowed"] is not None:
        v = torch.arange(V, device=z.device)
        z = torch.where(((s["allowed"][:, v >> 5] >> (v & 31)) & 1) != 0, z, torch.full_like(z, -math.inf))
    return z


def _plain_pick(z):
    most = z.amax(1, keepdim=True)
    token = (z == most).int().argmax(1)                # the first of them
    some = most != -math.inf
    rest = torch.exp(z - torch.where(some, most, torch.zeros_like(most))).scatter_(1, token[:, None], 0.0).sum(1)
    none = ~some[:, 0]
    return torch.where(none, torch.full_like(token, -1), token).to(torch.int32), torch.where(none, torch.full_like(rest, -math.inf), -torch.log1p(rest))


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "quantize":
        return _plain_quantize(state)
    if op == "logits":
        return _plain_logits(state)
    z = _plain_ruled(state)
    return z.to(state["z"].dtype) if op == "rules" else _plain_pick(z)


def work(case):
    op, V, e = case["op"], case["V"], BYTES[case["dtype"]]
    if op in ("quantize", "logits"):
        d = case["d"]
        q4 = V * d // 2 + V * -(-d // case["group"]) * 2
        if op == "quantize":                           # the weights in, their four bits and what they stand for out
            return {"bytes": 2 * V * d * e + q4, "flops": 4 * V * d}
        T = case["T"]
        return {"bytes": q4 + T * d * e + 4 * T * V, "flops": 2 * T * V * d}
    T = case["T"]
    inputs = T * V * e + 4 * T * case["H"] + 8 * T * case["B"] + 20 * T + (T * V // 8 if case["grammar"] else 0)
    return {"bytes": inputs + (T * V * e if op == "rules" else 8 * T), "flops": (4 if op == "rules" else 8) * T * V}


def _exact_quantize(case, seed):
    W = _weights(case, seed)["W"]
    out, group = torch.empty(W.shape, dtype=torch.float64, device=W.device), case["group"]
    for a in range(0, case["d"], group):
        w = W[:, a:a + group].double()
        largest = torch.maximum(w.max(1).values, -w.min(1).values)
        part, _ = torch.frexp(largest / 7)             # in [1/2, 1)
        one = 2 ** SCALE_BITS[case["scale"]]
        scale = torch.round(part * one) / one * (largest / 7 / part)
        steps = w / scale[:, None]
        below = torch.floor(steps)
        over = steps - below
        up = (over > 0.5) | ((over == 0.5) & (below % 2 != 0))
        out[:, a:a + group] = (below + up.double()) * scale[:, None]
    return out


def _exact_logits(case, seed):
    s = _head(case, seed)
    T, d, V = case["T"], case["d"], case["V"]
    x, out, dev = s["x"].double(), torch.empty((T, V), dtype=torch.float64, device="cuda"), "cuda"
    i = torch.arange(d, device=dev)
    inner = i % 128
    word, e = (inner // 8 % 4) * 64 + inner // 32, inner % 8                     # of a row of a tile: without the row's 4 words each
    nibble = e // 2 + 4 * (e % 2)
    for v0 in range(0, V, 16384):
        v = torch.arange(v0, min(V, v0 + 16384), device=dev)
        tile, row = v // 16, v % 16
        byte = s["codes"][tile[:, None], (i // 128)[None, :], (4 * (word[None, :] + 4 * row[:, None]) + (nibble // 2)[None, :])]
        q = ((byte >> (4 * (nibble % 2)).to(torch.uint8)[None, :]) & 15).double() - 8
        w = q * s["scales"][tile[:, None], (i // case["group"])[None, :], row[:, None]].double()
        out[:, v0:v0 + len(v)] = x.matmul(w.t())
    return out


def _exact_ruled(case, seed):
    s = _logit_inputs(case, seed)
    z, V = s["z"].double(), case["V"]
    for t in range(case["T"]):
        n, p = int(s["past_len"][t]), int(s["prompt_len"][t])
        past = s["past"][t, :n].long()
        seen = torch.unique(past)
        v = z[t, seen]
        rho = s["repetition"][t].double()
        z[t, seen] = torch.where(v > 0, v / rho, v * rho)
        token, count = torch.unique(past[p:], return_counts=True)
        z[t, token] -= s["frequency"][t].double() * count + s["presence"][t].double()
        if s["bias_ids"] is not None:
            has = s["bias_ids"][t] >= 0
            z[t].index_add_(0, s["bias_ids"][t][has].long(), s["bias_values"][t][has].double())
        if s["allowed"] is not None:
            words = s["allowed"][t].long() & 0xFFFFFFFF
            bits = (words[:, None] // 2 ** torch.arange(32, device=z.device)[None, :]) % 2
            z[t].masked_fill_(bits.reshape(-1)[:V] == 0, -math.inf)
    return z


def exact(case, seed):
    op = case["op"]
    if op == "quantize":
        return _exact_quantize(case, seed)
    if op == "logits":
        return _exact_logits(case, seed)
    z = _exact_ruled(case, seed)
    if op == "rules":
        return z
    most = z.max(1).values
    none = most == -math.inf
    first = torch.arange(case["V"], device=z.device).expand_as(z).masked_fill(z != most[:, None], case["V"]).min(1).values
    rest = z.scatter(1, first[:, None], -math.inf)     # without the token itself
    least = torch.logsumexp(rest, 1) - most
    return torch.where(none, -1, first).to(torch.int32), torch.where(none, most, -torch.log1p(torch.exp(least)))
