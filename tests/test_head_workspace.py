"""A head call's workspace grows with the rows: one that is sized for a program's largest batch serves every smaller one; what the binding refuses to take
for one, before anything is enqueued; and which strides it hands on (no GPU needed)."""
import itertools

import pytest
import torch

from paper_2603_21365_amd import tide_route as tr

SHAPES = [(4096, 128000), (768, 1147), (64, 300), (100, 50000), (8192, 18225), (1024, 1000), (8, 1), (16384, 32003)]


@pytest.mark.parametrize("d,V", SHAPES)
@pytest.mark.parametrize("dtype", [tr.F32, tr.F16, tr.BF16])
def test_more_rows_never_need_less(dtype, d, V):
    for K, kind in itertools.product((0, 32), ({}, {"gradient": True}, {"gradient": True, "wide": True})):
        most = 0
        for T in itertools.chain(range(0, 1400), range(1400, 9000, 37), (16384, 70000, 300000, 1 << 20)):
            if T * V > 1 << 37:
                continue
            need = tr.head_workspace_bytes(dtype, T, d, V, K, **kind)
            assert need >= most > 0 or most == 0, f"T={T} K={K} {kind}: {need} bytes, fewer rows {most}"
            most = need


class Stand(torch.Tensor):
    """A tensor that says it is on a GPU, for checks that come before any use of it."""
    is_cuda = True
    device = torch.device("cuda", 0)


def stand(t):
    return t.as_subclass(Stand)


@pytest.mark.parametrize("bad", [torch.empty(1, dtype=torch.uint8).expand(1 << 20), torch.empty(1 << 21, dtype=torch.uint8)[::2], torch.empty(1 << 20, dtype=torch.float32)])
def test_a_workspace_whose_bytes_are_not_its_elements_is_refused(bad):
    x = stand(torch.empty(4, 64))
    ok = stand(torch.empty(1 << 20, dtype=torch.uint8))
    assert tr._head_scratch(x, 4, 64, 100, 0, False, ok)[1] == 1 << 20 and tr._scratch(ok, 64, x.device)[1] == 1 << 20
    with pytest.raises(ValueError, match="workspace"):
        tr._head_scratch(x, 4, 64, 100, 0, False, stand(bad))
    with pytest.raises(ValueError, match="workspace"):
        tr._scratch(stand(bad), 64, x.device)


def test_a_workspace_of_another_device_is_refused():
    x = stand(torch.empty(4, 64))
    with pytest.raises(ValueError, match="workspace"):
        tr._head_scratch(x, 4, 64, 100, 0, False, torch.empty(1 << 20, dtype=torch.uint8))

    class Other(Stand):
        device = torch.device("cuda", 1)
    with pytest.raises(ValueError, match="workspace"):
        tr._head_scratch(x, 4, 64, 100, 0, False, torch.empty(1 << 20, dtype=torch.uint8).as_subclass(Other))


def test_one_row_has_no_stride():
    """The last token of a long sequence: its row's stride is the sequence's length, which no call would take between rows."""
    last = stand(torch.empty(1, 2000, 4096, dtype=torch.bfloat16))[:, -1]
    W = stand(torch.empty(3, 4096, dtype=torch.bfloat16))
    assert last.stride(0) > 1 << 22
    T, d, V, rows = tr._head_args(last, W)
    assert (T, d, V, rows[5], rows[7]) == (1, 4096, 3, 4096, 4096)
    assert tr._head_args(W, last)[3][7] == 4096
    pair = stand(torch.empty(2, 70, dtype=torch.bfloat16))[:, :64]
    assert tr._head_args(pair, pair)[3][5] == tr._head_args(pair, pair)[3][7] == 70


def test_two_planes_are_asked_for_with_the_type():
    """dtype | TIDE_HEAD_WIDE: another workspace above 64 rows of a 16-bit type, the same elsewhere; no type of a forward call."""
    size = lambda dtype, T, wide: tr.head_workspace_bytes(dtype, T, 512, 5000, gradient=True, wide=wide)
    for dtype in (tr.F16, tr.BF16):
        assert size(dtype, 200, True) > size(dtype, 200, False) and size(dtype, 64, True) == size(dtype, 64, False)
    assert size(tr.F32, 200, True) == size(tr.F32, 200, False)
    lib, fake = tr.load_library(), 0x100000
    wide = tr.BF16 | tr.HEAD_WIDE
    assert lib.tide_head_workspace_bytes(wide, 200, 512, 5000, 0, 1) == size(tr.BF16, 200, True)
    assert lib.tide_head_workspace_bytes(wide, 200, 512, 5000, 0, 0) == 0 and "dtype" in tr.last_error()
    assert lib.tide_head_workspace_bytes(3 | tr.HEAD_WIDE, 200, 512, 5000, 0, 1) == 0 and "dtype 3" in tr.last_error()
    assert lib.tide_head_loss(fake, wide, 4, 64, 100, 64, fake, 64, fake, fake, fake, fake, 0, None) == -1 and "dtype" in tr.last_error()
