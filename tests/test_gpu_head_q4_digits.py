"""Rows under an LM head in four bits: what large columns and wide scales leave of a logit's digits."""
import pytest
import torch

from paper_2603_21365_amd import tide_route as tr
from test_gpu_head_q4 import DTYPES, SCALES, generator, packed

pytestmark = pytest.mark.gpu

TS = (1, 3, 16, 20, 70, 200)           # rows in LDS, and rows that are laid out


def weights(codes, scales, group, d):
    return scales.double().repeat_interleave(group, dim=1)[:, :d] * (codes.double() - 8)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype,large", [("f32", 2.0 ** 40), ("f32", 2.0 ** 25 - 2), ("f16", 61440.0), ("bf16", 2.0 ** 40)])
def test_columns_without_weight_take_no_digits(dtype, large, group):
    """Half of the columns are large and have no weight (code 8): they add nothing, neither to a logit nor to its roundings.  What is left, integers below 5 times up to 8 and powers
    of two, is exact: 2^4 * 2^10 columns times 2^5, in steps of 2^-2."""
    V, d = 70, 1000
    g = generator(group)
    codes = torch.randint(0, 16, (V, d), generator=g).to(torch.uint8)
    codes[:, ::2] = 8
    scales = torch.pow(2.0, torch.randint(-2, 3, (V, -(-d // group)), generator=g).float())
    w = weights(codes, scales, group, d)
    head = packed(codes, scales.to(torch.bfloat16))
    for T in TS:
        x = torch.randint(-4, 5, (T, d), generator=g).double()
        want = x[:, 1::2] @ w[:, 1::2].T
        x[:, ::2] = large
        x[T // 2, ::4] = -large
        got = tr.head_logits_q4(x.to(DTYPES[dtype]).cuda(), *head, V, group)
        assert torch.equal(got.cpu().double(), want), f"T={T}: {(got.cpu().double() - want).abs().max()}"


@pytest.mark.parametrize("outliers", [False, True])
@pytest.mark.parametrize("scale", ["bf16", "f16"])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_digits_of_random_rows(dtype, group, scale, outliers):
    """A group's sum has `group` terms (fp32 rows: three times as many), added up with a rounding of at most 2^-23 of the sum so far each; a row's sum has one term a group.  The
    roundings are as good as independent, and sums so far of terms of either sign are no larger than the whole in the mean square: an error of 2^-23 sqrt(terms + groups) of the logits.  Columns that are 5000
    times as large and have no weight do not change that."""
    V, d, T = 300, 777, 40
    g = generator(group)
    codes = torch.randint(1, 16, (V, d), generator=g).to(torch.uint8)
    x = torch.randn((T, d), generator=g)
    if outliers:
        columns = torch.randperm(d, generator=g)[:12]
        codes[:, columns] = 8
        x[:, columns] *= 5000.0
    scales = (0.01 + torch.rand((V, -(-d // group)), generator=g)).to(SCALES[scale])
    x = x.to(DTYPES[dtype])
    want = x.double() @ weights(codes, scales, group, d).T
    head = packed(codes, scales)
    bound = 2.0 ** -23 * (group * (3 if dtype == "f32" else 1) + scales.shape[1]) ** 0.5 * want.square().mean().sqrt()
    for rows in (slice(0, 1), slice(0, 16), slice(0, T)):
        off = tr.head_logits_q4(x[rows].contiguous().cuda(), *head, V, group).cpu().double() - want[rows]
        assert off.square().mean().sqrt() <= bound, f"{rows}: {off.square().mean().sqrt() / bound} of the bound"


@pytest.mark.parametrize("T", [4, 40])
@pytest.mark.parametrize("scale", ["bf16", "f16"])
def test_every_bit_of_a_scale_counts(scale, T):
    """Rows with a one in one column: the logits are the weights, 8 or 11 bits times 4."""
    V, d, group = 200, 300, 32
    g = generator(T)
    codes = torch.randint(0, 16, (V, d), generator=g).to(torch.uint8)
    scales = (0.01 + torch.rand((V, -(-d // group)), generator=g)).to(SCALES[scale])
    w = weights(codes, scales, group, d)
    at = torch.randint(0, d, (T,), generator=g)
    for dtype in DTYPES.values():
        x = torch.zeros((T, d), dtype=dtype)
        x[torch.arange(T), at] = 1.0
        got = tr.head_logits_q4(x.cuda(), *packed(codes, scales), V, group)
        assert torch.equal(got.cpu().double(), w[:, at].T)


@pytest.mark.parametrize("T", [4, 40])
def test_every_bit_of_a_fp32_value_counts(T):
    """One value of 24 bits a row: its first bf16 term times the weight is exact, so is the sum of the others', and their sum is rounded once."""
    V, d, group = 100, 200, 64
    g = generator(T)
    codes = torch.randint(0, 16, (V, d), generator=g).to(torch.uint8)
    scales = torch.pow(2.0, torch.randint(-2, 3, (V, -(-d // group)), generator=g).float())
    at = torch.randint(0, d, (T,), generator=g)
    x = torch.zeros((T, d))
    x[torch.arange(T), at] = torch.randn(T, generator=g)
    got = tr.head_logits_q4(x.cuda(), *packed(codes, scales.to(torch.bfloat16)), V, group)
    assert torch.equal(got.cpu(), (x.double() @ weights(codes, scales, group, d).T).float())


@pytest.mark.parametrize("T,d", [(16, 8192), (3, 16384)])
def test_few_rows_in_parts_of_the_columns_in_a_graph(T, d):
    """The parts' sums are in the workspace, which a second launch adds up: it keeps nothing from one replay to the next."""
    V, group = 300, 64
    g = generator(d)
    codes = torch.randint(0, 256, (-(-V // 16), d // 128, 1024), generator=g).to(torch.uint8).cuda()
    scales = torch.ones((codes.shape[0], d // group, 16), dtype=torch.bfloat16, device="cuda")
    w = tr.head_dequantize_q4(codes, scales, V, d, torch.float32, group).cpu().double()
    need = tr.head_logits_q4_bytes(tr.F32, T, d, V)
    assert need > 0
    x, out, space = torch.zeros((T, d), device="cuda"), torch.empty((T, V), device="cuda"), torch.empty(need, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tr.head_logits_q4(x, codes, scales, V, group, out=out, workspace=space)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            tr.head_logits_q4(x, codes, scales, V, group, out=out, workspace=space)
    for _ in range(4):
        x.copy_(torch.randint(-2, 3, (T, d), generator=g))
        out.fill_(0.0), space.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu().double(), x.cpu().double() @ w.T)      # 2 * 8 * 16384 in steps of 1/16: 22 bits
