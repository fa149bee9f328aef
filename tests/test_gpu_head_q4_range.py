"""Rows under an LM head in four bits at the upper end of the values' range."""
import pytest
import torch

from paper_2603_21365_amd import tide_route as tr
from test_gpu_head_q4 import DTYPES, generator, packed

pytestmark = pytest.mark.gpu


def weights(codes, scales, group, d):
    return scales.double().repeat_interleave(group, dim=1)[:, :d] * (codes.double() - 8)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("T", [6, 30])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_magnitudes_around_the_largest(dtype, T, group):
    """Rows whose magnitudes in a group add up to 2^126: no logit of theirs is a number, whatever the codes are, and no other row's is touched.  Below that the logits are the products
    (scales of 2^-10: none is beyond fp32)."""
    V, d = 50, 260
    g = generator(T)
    codes = torch.randint(0, 16, (V, d), generator=g).to(torch.uint8)
    scales = torch.full((V, -(-d // group)), 2.0 ** -10)
    w, head = weights(codes, scales, group, d), packed(codes, scales.to(torch.bfloat16))
    x = torch.randint(-4, 5, (T, d), generator=g).float()
    most = (2 - 2.0 ** -7) * 2.0 ** 125                 # the largest bf16 value below 2^126
    x[0], x[1], x[2], x[3], x[4] = 0, 0, 0, 0, 0
    x[0, 7] = 2.0 ** 126
    x[1, 259] = -(2 - 2.0 ** -7) * 2.0 ** 127           # the lowest bf16 value
    x[2, 130], x[2, 141] = 2.0 ** 125, -2.0 ** 125      # (they cancel)
    x[3, 130] = -most
    x[4, 31], x[4, 128] = most, most                    # (two groups)
    for rows in (x, x[[3, 0, 4, 5]]):
        got = tr.head_logits_q4(rows.to(DTYPES[dtype]).cuda(), *head, V, group).cpu()
        bad = torch.tensor([i in (0, 1, 2) if rows is x else i == 1 for i in range(len(rows))])
        assert torch.isnan(got[bad]).all(), got[bad]
        assert torch.equal(got[~bad].double(), rows[~bad].double() @ w.T)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_an_infinity_in_any_column_even_one_without_weight(dtype, group):
    """Row i has one in column i, whose code is 8 for every second token: none of the row's logits is a number, all of the clean rows' are what they were."""
    V, d = 37, 200
    g = generator(group)
    codes = torch.randint(0, 16, (V, d), generator=g).to(torch.uint8)
    codes[::2] = 8
    scales = torch.pow(2.0, torch.randint(-2, 3, (V, -(-d // group)), generator=g).float())
    w, head = weights(codes, scales, group, d), packed(codes, scales.to(torch.bfloat16))
    x = torch.randint(-4, 5, (2 * d, d), generator=g).float()
    want = x.double() @ w.T
    x[torch.arange(0, 2 * d, 2), torch.arange(d)] = float("inf")
    x[2 * 150, 150] = float("nan")
    rows = x.to(DTYPES[dtype]).cuda()
    for got in (tr.head_logits_q4(rows, *head, V, group), torch.cat([tr.head_logits_q4(part, *head, V, group) for part in rows.split(13)])):
        assert torch.isnan(got[::2]).all() and torch.equal(got[1::2].cpu().double(), want[1::2])


@pytest.mark.parametrize("T", [4194303, 4194304])
def test_the_most_rows(T):
    V, d = 2, 3
    codes, scales = torch.tensor([[9, 3, 15], [0, 8, 10]], dtype=torch.uint8), torch.tensor([[2.0], [0.5]])
    x = torch.randint(-4, 5, (T, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    got = tr.head_logits_q4(x, *packed(codes, scales.to(torch.bfloat16)), V, 32)
    assert torch.equal(got, (x.float()[:, None, :] * weights(codes, scales, 32, d).float().cuda()).sum(2))
