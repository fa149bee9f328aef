"""The most rows that the rules of decoding take."""
import pytest
import torch

from paper_2603_21365_amd import tide_route as tr

pytestmark = pytest.mark.gpu


def test_the_most_rows():
    T = 4194303
    z = (torch.arange(T, device="cuda") % 1000).float()[:, None]
    out = tr.logit_rules(z, past=torch.zeros((T, 1), dtype=torch.int32, device="cuda"), repetition=torch.full((T,), 2.0, device="cuda"))
    assert torch.equal(out, z / 2)
    token, log_prob = tr.logit_pick(z)
    assert int(token.abs().max()) == 0 and int((log_prob != 0).sum()) == 0
