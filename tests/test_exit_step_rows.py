"""Which rows a training step at the exits counts: those that the head operators give a loss (no GPU needed; the operators are stood in for)."""
import pytest
import torch

from paper_2603_21365_amd import exit_tuning

T, d, V, K = 6, 4, 10, 2


@pytest.fixture
def step(monkeypatch):
    """exit_step on stand-ins of the operators: a loss of one for each row it is to count, and the upstream gradient that it hands on."""
    seen = {}

    class Operators:
        exit_project = staticmethod(lambda *a: torch.zeros(T, d))
        exit_project_grad = staticmethod(lambda *a: (torch.zeros(T, d), torch.zeros(d)))

        @staticmethod
        def head_loss(rows, head, target):
            return ((target >= 0) & (target < V)).float(), torch.zeros(T)

        @staticmethod
        def head_distill(rows, head, values, ids, tau):
            return seen["counts"].float(), torch.zeros(T), torch.zeros(T, K)

        @staticmethod
        def head_loss_grad(rows, head, target, lse, grad_loss):
            seen["grad_loss"] = grad_loss
            return torch.zeros(T, d), torch.zeros(V, d)

        @staticmethod
        def head_distill_grad(rows, head, values, ids, tau, lse, grad_loss):
            seen["grad_loss"] = grad_loss
            return torch.zeros(T, d), torch.zeros(V, d)

    monkeypatch.setattr(exit_tuning, "tr", Operators)

    def run(counts, **taught_by):
        seen["counts"] = counts
        out = exit_tuning.exit_step(None, None, None, None, None, 1e-6, torch.zeros(V, d), **taught_by)
        return out, seen["grad_loss"]
    return run


def test_rows_of_a_teacher_without_an_entry_are_not_counted(step):
    inf = float("inf")
    ids = torch.tensor([[1, 2], [-1, -1], [V, V + 7], [3, 4], [5, V], [-1, 9]], dtype=torch.int32)
    values = torch.tensor([[0.0, 1.0], [0.0, 0.0], [0.0, 0.0], [-inf, -inf], [-inf, 1.0], [2.0, 0.5]])
    counts = torch.tensor([True, False, False, False, False, True])
    out, grad_loss = step(counts, teacher=(values, ids))
    assert out.mean == 1.0
    assert torch.equal(grad_loss, torch.where(counts, 0.5, 0.0))


def test_rows_without_a_target_are_not_counted(step):
    target = torch.tensor([0, -1, V, V - 1, -2147483648, 5], dtype=torch.int32)
    counts = torch.tensor([True, False, False, True, False, True])
    out, grad_loss = step(counts, target=target)
    assert out.mean == 1.0
    assert torch.allclose(grad_loss, torch.where(counts, 1 / 3, 0.0))
