"""A head call's workspace grows with the rows: one that is sized for a program's largest batch serves every smaller one (no GPU needed)."""
import itertools

import pytest

from paper_2603_21365_amd import tide_route as tr

SHAPES = [(4096, 128000), (768, 1147), (64, 300), (100, 50000), (8192, 18225), (1024, 1000), (8, 1), (16384, 32003)]


@pytest.mark.parametrize("d,V", SHAPES)
@pytest.mark.parametrize("dtype", [tr.F32, tr.F16, tr.BF16])
def test_more_rows_never_need_less(dtype, d, V):
    for K, gradient in itertools.product((0, 32), (False, True)):
        most = 0
        for T in itertools.chain(range(0, 1400), range(1400, 9000, 37), (16384, 70000, 300000, 1 << 20)):
            if T * V > 1 << 37:
                continue
            need = tr.head_workspace_bytes(dtype, T, d, V, K, gradient=gradient)
            assert need >= most > 0 or most == 0, f"T={T} K={K} gradient={gradient}: {need} bytes, fewer rows {most}"
            most = need
