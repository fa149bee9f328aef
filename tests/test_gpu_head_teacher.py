"""Teachers that are broken or at the ends of their type.  Hidden states of zero under a head of unit rows: z = 0, lse = log V, and dx IS the gradient to
the logits, g tau (1 / V - q), so a teacher's probabilities can be read off."""
import math

import pytest

pytestmark = pytest.mark.gpu

V = 64
E = 2.0 ** -24


@pytest.fixture(scope="module")
def tr():
    import torch
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    tide_route.load_library()
    return tide_route


def distill(tr, values, tau):
    """(loss, dx, dW) of rows of zeros under the unit head for a teacher's values at the tokens 0 .. K - 1."""
    import torch
    T, K = values.shape
    x, W = torch.zeros(T, V, device="cuda"), torch.eye(V, device="cuda")
    ids = torch.arange(K, device="cuda", dtype=torch.int32).repeat(T, 1).contiguous()
    ones = torch.ones(T, device="cuda")
    loss, lse, _ = tr.head_distill(x, W, values, ids, tau)
    dx, dW = tr.head_distill_grad(x, W, values, ids, tau, lse, ones)
    torch.cuda.synchronize()
    return loss, dx, dW


def exact(values, tau):
    import torch
    q = torch.softmax(values.double() / tau, 1)
    entropy = -torch.where(q > 0, q * torch.log(q.clamp(min=1e-300)), 0.0).sum(1)
    dx = torch.full((values.shape[0], V), tau / V, dtype=torch.float64, device="cuda")
    dx[:, :values.shape[1]] -= tau * q
    return q, tau * tau * (math.log(V) - entropy), dx


@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_a_broken_teacher_is_a_broken_loss(tr, bad):
    """A NaN or +inf among a row's values makes that row's loss NaN, as it makes its gradient, and leaves the other rows'."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    values = torch.randn(5, 8, generator=g, device="cuda")
    good, good_dx, _ = distill(tr, values, 2.0)
    values[2, 3] = float(bad)
    print(f"[gpu-case] broken teacher {bad}", flush=True)
    loss, dx, _ = distill(tr, values, 2.0)
    rows = [0, 1, 3, 4]
    assert loss[2].isnan() and dx[2].isnan().any()
    assert torch.equal(loss[rows], good[rows]) and torch.equal(dx[rows], good_dx[rows])


@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0 ** -7])
def test_a_teacher_of_the_lowest_values(tr, tau):
    """Rows whose values are all the type's lowest one are uniform; among others such a value has no weight.  Bounds: six roundings of a probability, 16 of a loss."""
    import torch
    low = torch.finfo(torch.float32).min
    values = torch.zeros(4, 8, device="cuda")
    values[1] = low
    values[2, 3:] = low
    values[3] = torch.finfo(torch.float32).max
    print(f"[gpu-case] lowest values, tau {tau}", flush=True)
    loss, dx, _ = distill(tr, values, tau)
    q, want, want_dx = exact(values, tau)
    assert (q[[0, 1, 3]] == 1 / 8).all() and (q[2, 3:] == 0).all()
    assert ((loss.double() - want).abs() <= 16 * E * tau * tau * math.log(V)).all()
    assert ((dx.double() - want_dx).abs() <= 6 * E * tau * (q.amax(1, keepdim=True) + 1 / V) + 2.0 ** -22 * want_dx.abs()).all()


def test_a_teacher_of_large_values_at_a_small_temperature(tr):
    """Probabilities hang on the values' differences: 1000 + k / 512 at tau = 0.0077 are about exp(k / 4) to a dozen roundings, not to 2^-24 of 130000.
    (The difference, its quotient and both exponentials' arguments, each below 8 here, and the sum's: (4 * 8 + 12) e.)"""
    import torch
    tau = torch.tensor(0.0077, dtype=torch.float32).item()
    values = (1000 + torch.arange(32, device="cuda").float().flip(0) / 512)[None].repeat(3, 1).contiguous()
    values[1] = -values[1]
    values[2] = values[2, torch.randperm(32, device="cuda")]
    print("[gpu-case] large values, small temperature", flush=True)
    loss, dx, _ = distill(tr, values, tau)
    q, want, want_dx = exact(values, tau)
    tol = (4 * 8 + 12) * E
    assert ((dx.double() - want_dx).abs() <= tau * (tol * q.amax(1, keepdim=True) + 16 * E / V) + 2.0 ** -22 * want_dx.abs()).all()
    assert ((loss.double() - want).abs() <= 4 * tol * tau * tau * math.log(V)).all()
