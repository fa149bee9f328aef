"""The limits of the answer operators as the host checks them: what the documents allow is not refused further on, and what they do not is named (no GPU needed)."""
import pytest

from paper_2603_21365_amd import tide_route as tr
from test_answer_arguments import UNSUPPORTED, pick, rules


@pytest.mark.parametrize("call", [rules, pick])
def test_a_row_more_than_a_launch_has(call):
    assert call(T=1 << 22) == UNSUPPORTED and "T = 4194304 exceeds 4194303" in tr.last_error()


def test_no_workspace_is_named_for_rows_that_are_refused():
    for V in (1, 16384, 16385):
        assert tr.logit_pick_bytes(1 << 22, V) == 0 and "unsupported" in tr.last_error()
    assert tr.logit_pick_bytes((1 << 22) - 1, 1) == 0 and tr.last_error() == ""
