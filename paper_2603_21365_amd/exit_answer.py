"""One decode step at the exits: every token's exit is selected, the row it exits with is projected and scored under an LM head in four bits, and the rules of
decoding give its next token.

    python -m paper_2603_21365_amd.exit_answer        a few steps on synthetic states
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import tide_route as tr


@dataclass
class Head:
    """An LM head in four bits."""
    codes: torch.Tensor
    scales: torch.Tensor
    V: int
    group: int = 128

    @classmethod
    def of(cls, W, group=128, scale_dtype=torch.bfloat16) -> "Head":
        """Of the weights W [V,d]."""
        return cls(*tr.head_quantize_q4(W, group, scale_dtype=scale_dtype), W.shape[0], group)

    def logits(self, rows) -> torch.Tensor:
        return tr.head_logits_q4(rows, self.codes, self.scales, self.V, self.group)


@dataclass
class Routers:
    """What select_exit_packed takes beside the states."""
    packed: torch.Tensor
    eps: float
    b1: torch.Tensor | None
    w2: torch.Tensor
    b2: object
    threshold: object
    layer_ids: list
    min_layer: int
    n_layers: int


@dataclass
class ExitAnswer:
    """What a step gives."""
    token: torch.Tensor              # int32 [T], -1 where the rules leave none
    log_prob: torch.Tensor           # f32 [T]
    exit_layer: torch.Tensor         # int32 [T]


def answer_step(hidden, final_hidden, routers: Routers, norm_gain, eps, head: Head, **rules) -> ExitAnswer:
    """hidden [C,T,d], final_hidden [T,d] (the last layer's states, for tokens that no router lets exit), norm_gain f32 [d] | None and eps of the final norm;
    ``rules``: logit_pick's past, penalties, biases and mask.  Inference only: no gradients."""
    r = routers
    exit_layer, _, _ = tr.select_exit_packed(hidden, r.packed, r.eps, r.b1, r.w2, r.b2, r.threshold, r.layer_ids, r.min_layer, r.n_layers, d=hidden.shape[-1],
                                             want_logits=False, want_mask=False)
    rows = tr.exit_project(hidden, final_hidden, exit_layer, r.layer_ids, norm_gain, eps)
    token, log_prob = tr.logit_pick(head.logits(rows), **rules)
    return ExitAnswer(token, log_prob, exit_layer)


def main(steps: int = 8, T: int = 4, d: int = 1024, V: int = 8000, C: int = 4, group: int = 64) -> list:
    """Generates ``steps`` tokens for each of T sequences: random states, and a past that is penalised.  Returns the tokens of each step."""
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    ids = [4 * c + 3 for c in range(C)]
    packed = tr.router_pack(tr.BF16, None, randn(C, d, 128) * d ** -0.5)
    routers = Routers(packed, 1e-6, None, randn(C, 128) * 0.3, 0.0, 0.5, ids, 0, 4 * C)
    head = Head.of((randn(V, d) * (1.5 / d ** 0.5)).to(torch.bfloat16), group)
    gain = torch.ones(d, device="cuda")
    past = torch.full((T, steps), -1, dtype=torch.int32, device="cuda")
    row = lambda x: torch.full((T,), x, device="cuda")
    tokens = []
    for step in range(steps):
        final = randn(T, d)
        hidden = torch.stack([final + (1.0 - 0.2 * c) * randn(T, d) for c in range(C)]).to(torch.bfloat16)
        answer = answer_step(hidden, final.to(torch.bfloat16), routers, gain, 1e-6, head, past=past, repetition=row(1.2), presence=row(0.3), frequency=row(0.1))
        past[:, step] = answer.token
        tokens.append(answer.token.tolist())
    return tokens


if __name__ == "__main__":
    for tokens in main():
        print(" ".join(f"{t:6d}" for t in tokens))
