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
