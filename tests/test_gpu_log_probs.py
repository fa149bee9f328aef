"""The digits of log-probabilities."""
import pytest
import torch

from paper_2603_21365_amd import tide_route as tr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [2, 3, 9, 5000, 40000])
def test_a_term_of_the_sum_keeps_its_digits(V):
    """One other token, at a distance of up to 80: the log-probability is -log1p(exp(-distance)).  exp2 is good to 2^-23, the correction for its argument's rounding is rounded once
    more, 2^-24, and log1p is good to 2^-22: less than 2^-21 together."""
    T = 300
    g = torch.Generator().manual_seed(V)
    off = 0.5 + 79.5 * torch.rand(T, generator=g)
    z = torch.full((T, V), -300.0)
    at = torch.argsort(torch.rand((T, V), generator=g), 1)[:, :2]
    z.scatter_(1, at[:, :1], 0.0).scatter_(1, at[:, 1:], -off[:, None])
    token, log_prob = tr.logit_pick(z.cuda())
    assert torch.equal(token.cpu().long(), at[:, 0])
    want = -torch.log1p(torch.exp(-off.double()))
    rel = ((log_prob.cpu().double() - want) / want).abs()
    assert rel.max() <= 2.0 ** -21, f"{rel.max() * 2 ** 21} of the bound, at {off[rel.argmax()]}"


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_distances_beyond_all_range(dtype):
    """The widest distance that the type has, equal lowest values and -inf: no term is anything but zero or one."""
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    for V in (2, 5, 1030, 70000):
        z = torch.full((5, V), low, dtype=dtype)
        z[0, 1] = high
        z[2] = -float("inf")
        z[2, 0] = low
        z[3, 0] = -float("inf")
        z[4] = -float("inf")
        z[4, 1] = high
        token, log_prob = (a.cpu() for a in tr.logit_pick(z.cuda()))
        assert token.tolist() == [1, 0, 0, 1, 1]
        want = torch.tensor([0.0, -torch.log(torch.tensor(float(V), dtype=torch.float64)), 0.0, -torch.log(torch.tensor(float(V - 1), dtype=torch.float64)), 0.0], dtype=torch.float64)
        assert (log_prob.double() - want).abs().max() <= 2.0 ** -21 * want.abs().max()       # (sums of ones are exact)
