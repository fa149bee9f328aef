"""One training step at the exits: the rows that tokens exit with are projected, scored under the LM head, and the gradients go back to the head, to the
final norm's gain and to the exited rows.  The head is taught the next tokens, or (``teacher``) the full depth's few largest logits.

    python -m paper_2603_21365_amd.exit_tuning        a few steps on synthetic states
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import tide_route as tr


@dataclass
class ExitStep:
    """What a step gives: the mean loss of its rows, each row's, and the gradients of the mean."""
    mean: torch.Tensor
    loss: torch.Tensor
    grad_rows: torch.Tensor          # [T, d] to the row each token exited with
    grad_gain: torch.Tensor          # [d] fp32
    grad_head: torch.Tensor          # [V, d]


def exit_step(hidden, final_hidden, exit_layer, layer_ids, norm_gain, eps, head, *, target=None, teacher=None, tau=1.0, loss_scale=1.0) -> ExitStep:
    """hidden [C,T,d], final_hidden [T,d], exit_layer int32 [T] (select_exit's), layer_ids host [C], norm_gain fp32 [d], head [V,d]; either
    target int32 [T] (negative: none) or teacher = (top_values f32 [T,K], top_ids int32 [T,K]).  The gradients carry ``loss_scale`` (against
    fp16's underflow); rows without a target or teacher count neither in the mean nor in the gradients."""
    rows = tr.exit_project(hidden, final_hidden, exit_layer, layer_ids, norm_gain, eps)
    if teacher is None:
        taught = (target >= 0) & (target < head.shape[0])
        loss, lse = tr.head_loss(rows, head, target)
    else:
        values, ids = teacher
        taught = ((ids >= 0) & (ids < head.shape[0]) & (values != -torch.inf)).any(1)      # the entries that head_distill counts
        loss, lse, _ = tr.head_distill(rows, head, *teacher, tau)
    count = taught.sum().clamp(min=1)
    grad_loss = taught.to(torch.float32) * (loss_scale / count)
    if teacher is None:
        grad_out, grad_head = tr.head_loss_grad(rows, head, target, lse, grad_loss)
    else:
        grad_out, grad_head = tr.head_distill_grad(rows, head, *teacher, tau, lse, grad_loss)
    grad_rows, grad_gain = tr.exit_project_grad(hidden, final_hidden, exit_layer, layer_ids, norm_gain, eps, grad_out)
    return ExitStep(loss.sum() / count, loss, grad_rows, grad_gain, grad_head)


def main(steps: int = 6, T: int = 512, d: int = 1024, V: int = 8000, C: int = 4, K: int = 16, tau: float = 2.0) -> list:
    """Distils the last layer's answers into exits at random checkpoints; returns the mean loss of each step."""
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    final = randn(T, d)
    hidden = torch.stack([final + (1.0 - 0.2 * c) * randn(T, d) for c in range(C)]).to(torch.bfloat16)
    final = final.to(torch.bfloat16)
    head = (randn(V, d) * (1.5 / d ** 0.5)).to(torch.bfloat16)
    gain, ids = torch.ones(d, device="cuda"), [4 * c + 3 for c in range(C)]
    exits = (4 * torch.randint(0, C, (T,), generator=g, device="cuda") + 3).to(torch.int32)
    nowhere = torch.full_like(exits, 4 * C)                # full depth: the teacher
    top = (tr.exit_project(hidden, final, nowhere, ids, gain, 1e-6).float() @ head.float().T).topk(K, dim=1)
    teacher = (top.values.contiguous(), top.indices.to(torch.int32).contiguous())
    weights, losses = head.float(), []
    for _ in range(steps):
        s = exit_step(hidden, final, exits, ids, gain, 1e-6, weights.to(torch.bfloat16), teacher=teacher, tau=tau)
        losses.append(s.mean.item())
        weights -= 5.0 * s.grad_head.float()
        gain -= 0.1 * s.grad_gain
    return losses


if __name__ == "__main__":
    print("mean loss by step:", " ".join(f"{x:.4f}" for x in main()))
