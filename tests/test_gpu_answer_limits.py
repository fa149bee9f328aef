"""The answer operators at the ends of their ranges: offsets that pass 32 bits, the widest rows, pasts whose counts pass 16 bits, the most biases, many rows in a graph."""
import pytest
import torch

from paper_2603_21365_amd import tide_route as tr

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def integers(low, high, shape, seed, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(low, high, shape, generator=g, device="cuda").to(dtype)


def lowest_of_largest(z):
    return [int((row == row.max()).nonzero()[0]) for row in z]


def packed(V, d, group, seed):
    """Codes and scales of one; the weights [V,d] they stand for come from head_dequantize_q4, which has tests of its own."""
    rows, blocks = -(-V // 16), -(-d // 128)
    codes = integers(0, 256, (rows, blocks, 1024), seed, torch.uint8)
    return codes, torch.ones((rows, -(-d // group), 16), dtype=torch.bfloat16, device="cuda")


@pytest.mark.parametrize("T,group", [(1, 64), (20, 128)])
def test_codes_beyond_2_to_the_31_bytes(T, group):
    """The last tokens' logits are those of a head that has only them.  (d = 1100 terms of up to 2 * 8 in steps of 1/16: 2^14.2 and 19 bits, exact in any order.)"""
    d, V = 1100, (1 << 22) + (1 << 19) + 37
    codes, scales = packed(V, d, group, 3)
    assert codes.numel() > 2 ** 31
    x = integers(-2, 3, (T, d), 4, torch.bfloat16)
    out = tr.head_logits_q4(x, codes, scales, V, group)
    for first in (0, 1 << 17, codes.shape[0] - 5):     # (codes past 2^30 and 2^31 bytes)
        tokens = min(16 * 5, V - 16 * first)
        want = tr.head_logits_q4(x, codes[first:first + 5].contiguous(), scales[first:first + 5].contiguous(), tokens, group)
        assert torch.equal(out[:, 16 * first:16 * first + tokens], want)
        w = tr.head_dequantize_q4(codes[first:first + 5].contiguous(), scales[first:first + 5].contiguous(), tokens, d, torch.float32, group)
        assert torch.equal(want.cpu().double(), x.cpu().double() @ w.cpu().double().T)


def test_weights_beyond_2_to_the_31_elements():
    d, V = 1100, (1 << 21) + 5
    W = integers(-7, 8, (V, d), 5, torch.bfloat16)
    assert W.numel() > 2 ** 31
    codes, scales = tr.head_quantize_q4(W, 64)
    back = tr.head_dequantize_q4(codes, scales, V, d, torch.bfloat16, 64)
    first = (V // 16 - 4) * 16
    part_codes, part_scales = tr.head_quantize_q4(W[first:].contiguous(), 64)
    assert torch.equal(codes[first // 16:], part_codes) and torch.equal(scales[first // 16:], part_scales)
    assert torch.equal(back[first:], tr.head_dequantize_q4(part_codes, part_scales, V - first, d, torch.bfloat16, 64))
    # integers of a group with a 7 or a -7 are its codes; hardly a group of 64 has none
    same = (back[first:] == W[first:]).float().mean()
    assert same > 0.9


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_logits_beyond_2_to_the_31(dtype):
    T, V = 1100, (1 << 21) + 5
    z = torch.zeros((T, V), dtype=DTYPES[dtype], device="cuda")
    assert z.numel() > 2 ** 31
    rows = [0, 7, 1023, 1099]
    for t in rows:
        z[t] = integers(-50, 51, (V,), 100 + t).to(z.dtype) / 8
    past = torch.full((T, 30), -1, dtype=torch.int32, device="cuda")
    past[:, :20] = integers(0, V, (T, 20), 6, torch.int32)
    c = dict(past=past, repetition=torch.full((T,), 1.5, device="cuda"), presence=torch.full((T,), 0.5, device="cuda"),
             bias_ids=integers(0, V, (T, 4), 7, torch.int32), bias_values=integers(20, 30, (T, 4), 8))
    at = torch.tensor(rows, device="cuda")
    few = {k: v[at].contiguous() for k, v in c.items()}
    want, (token, log_prob) = tr.logit_rules(z[at], **few), tr.logit_pick(z[at], **few)
    got = tr.logit_pick(z, **c)
    assert torch.equal(got[0][at], token) and (token >= 0).all()
    # some 2^21 terms a row, each rounded, added up by threads in sums of at most 2^10 and then of at most 2^11
    assert ((got[1][at] - log_prob).abs() <= 2.0 ** -24 * (2 ** 10 + 2 ** 11)).all()
    out = tr.logit_rules(z, **c, out=z)
    assert torch.equal(out[at], want)
    others = torch.tensor([1, 8, 1098], device="cuda")  # zeros: their biases are all that was added
    for t in others.tolist():
        assert int((out[t] != 0).sum()) == int(torch.unique(torch.cat([past[t, :20], c["bias_ids"][t]])).numel())


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_the_widest_rows(dtype, group):
    """d = 16384, in LDS or not: terms of up to 8 in steps of 1/16 (2 * 1.94 before the offset), 16384 of them below 2^17: 21 bits."""
    d, V = 16384, 100
    codes, scales = packed(V, d, group, 9)
    w = tr.head_dequantize_q4(codes, scales, V, d, torch.float32, group).cpu().double()
    for T in (1, 2, 3, 5, 9, 16, 17, 40):
        x = integers(-1, 2, (T, d), T)
        got = tr.head_logits_q4(x.to(DTYPES[dtype]), codes, scales, V, group)
        assert torch.equal(got.cpu().double(), x.cpu().double() @ w.T), f"T={T}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H", [32767, 32768, 70001])
def test_counts_around_16_bits(H, dtype):
    """A token that is all of a past, beside one that is in the prompt only, and none of its neighbours touched."""
    V, n = 70, H - 2
    z = integers(-20, 21, (2, V), 1).to(DTYPES[dtype])
    past = torch.full((2, H), 5, dtype=torch.int32, device="cuda")
    past[1, 0], past[1, 1] = 4, 6
    lengths, prompts = torch.tensor([H, n], dtype=torch.int32, device="cuda"), torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    two, zero = torch.full((2,), 2.0, device="cuda"), torch.zeros(2, device="cuda")
    frequency = torch.full((2,), 2.0 ** -12, device="cuda")
    c = dict(past=past, past_len=lengths, prompt_len=prompts, repetition=two, presence=zero + 0.5, frequency=frequency)
    rule = lambda a: torch.where(a > 0, a / 2, a * 2)
    want = z.float().clone()
    want[0, 5] = rule(want[0, 5]) - (H * 2.0 ** -12 + 0.5)
    want[1, 5] = rule(want[1, 5]) - ((n - 2) * 2.0 ** -12 + 0.5)
    want[1, 4], want[1, 6] = rule(want[1, 4]), rule(want[1, 6])
    # (integers and halves below 2^6 and multiples of 2^-12 below 2^5: 18 bits)
    assert torch.equal(tr.logit_rules(z, **c), want.to(z.dtype))
    token, _ = tr.logit_pick(z, **c)
    assert token.tolist() == lowest_of_largest(want)


@pytest.mark.parametrize("spread", [1, 3, 1000])
def test_the_most_biases(spread):
    """1024 entries on few tokens; sums of integers below 2^15 are exact in any order."""
    T, V, B = 3, 5000, 1024
    z = integers(-50, 51, (T, V), 2)
    ids, values = integers(0, spread, (T, B), 3, torch.int32) * 4, integers(-20, 21, (T, B), 4)
    want = z.clone().scatter_add_(1, ids.long(), values)
    assert torch.equal(tr.logit_rules(z, bias_ids=ids, bias_values=values), want)
    token, _ = tr.logit_pick(z, bias_ids=ids, bias_values=values)
    assert token.tolist() == lowest_of_largest(want)


@pytest.mark.parametrize("dtype,unit", [("f16", 2.0 ** -24), ("bf16", 2.0 ** -120), ("bf16", 2.0 ** 110), ("f32", 2.0 ** -100), ("f32", 2.0 ** 110)])
def test_tiny_and_huge_rows(dtype, unit):
    """Rows of integers times a power of two -- for fp16 the smallest one that it has -- have the integers' logits times that; all exact, as above."""
    V, d, group = 60, 200, 64
    codes, scales = packed(V, d, group, 13)
    w = tr.head_dequantize_q4(codes, scales, V, d, torch.float32, group).cpu().double()
    for T in (1, 4, 40):
        x = integers(-2, 3, (T, d), T)
        got = tr.head_logits_q4((x * unit).to(DTYPES[dtype]), codes, scales, V, group)
        assert torch.equal(got.cpu().double(), x.cpu().double() @ w.T * unit), f"T={T}"


def test_many_rows_in_graphs_with_workspaces_of_their_own():
    V, d, group = 300, 260, 64
    codes, scales = packed(V, d, group, 11)
    w = tr.head_dequantize_q4(codes, scales, V, d, torch.float32, group).cpu().double()
    cases = []
    side = torch.cuda.Stream()
    for T, dtype in ((40, torch.bfloat16), (130, torch.float16), (33, torch.float32)):
        x = integers(-2, 3, (T, d), T, dtype)
        space = torch.empty(tr.head_logits_q4_bytes({torch.float32: tr.F32, torch.float16: tr.F16, torch.bfloat16: tr.BF16}[dtype], T, d, V), dtype=torch.uint8, device="cuda")
        out = torch.empty((T, V), device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            tr.head_logits_q4(x, codes, scales, V, group, out=out, workspace=space)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                tr.head_logits_q4(x, codes, scales, V, group, out=out, workspace=space)
        cases.append((x, space, out, graph))
    for seed in range(4):
        for x, space, out, _ in cases:
            x.copy_(integers(-2, 3, tuple(x.shape), 50 + seed))
            out.fill_(0.0), space.fill_(255)
        torch.cuda.synchronize()
        for *_, graph in cases:
            graph.replay()
        torch.cuda.synchronize()
        for x, _, out, _ in cases:
            assert torch.equal(out, tr.head_logits_q4(x, codes, scales, V, group)) and torch.equal(out.cpu().double(), x.cpu().double() @ w.T)


@pytest.mark.parametrize("dtype,d,V", [("f32", 8192, 3001), ("f16", 8192, 500), ("bf16", 5120, 3001), ("f32", 1100, 70), ("bf16", 12288 + 77, 1)])
def test_columns_in_parts(dtype, d, V):
    """Few tokens under many columns, which several workgroups share, into rows with gaps: exact as above (2 * 8 * 12365 in steps of 1/16: 22 bits), and what lies between the rows stays."""
    codes, scales = packed(V, d, 64, d + V)
    w = tr.head_dequantize_q4(codes, scales, V, d, torch.float32, 64).cpu().double()
    for T in (2, 7, 16, 17, 50, 200):
        x = integers(-2, 3, (T, d + 3), T, DTYPES[dtype])[:, 1:1 + d]
        space = torch.full((tr.head_logits_q4_bytes({"f32": tr.F32, "f16": tr.F16, "bf16": tr.BF16}[dtype], T, d, V),), 255, dtype=torch.uint8, device="cuda")
        out = torch.full((T, V + 9), 7.0, device="cuda")
        tr.head_logits_q4(x, codes, scales, V, 64, out=out[:, 4:4 + V], workspace=space)
        assert torch.equal(out[:, 4:4 + V].cpu().double(), x.cpu().double() @ w.T), f"T={T}"
        assert (out[:, :4] == 7).all() and (out[:, 4 + V:] == 7).all()


def test_two_streams_at_once():
    V, d, group, T = 4000, 512, 32, 24
    codes, scales = packed(V, d, group, 12)
    xs = [integers(-2, 3, (T, d), 60 + i, torch.float16) for i in range(2)]
    want = [tr.head_logits_q4(x, codes, scales, V, group) for x in xs]
    picks = [tr.logit_pick(z) for z in want]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                z = tr.head_logits_q4(xs[i], codes, scales, V, group)
                got[i].append((z, tr.logit_pick(z)))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(z, want[i]) and torch.equal(p[0], picks[i][0]) and torch.equal(p[1], picks[i][1]) for z, p in got[i])
