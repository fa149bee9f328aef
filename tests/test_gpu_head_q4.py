"""The LM head in four bits on the GPU: its codes and scales against the definition in 64 bits, the values read back, rows scored under it."""
import numpy as np
import pytest
import torch

from paper_2603_21365_amd import tide_route as tr

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SCALES = {"f16": torch.float16, "bf16": torch.bfloat16}


def generator(seed):
    return torch.Generator().manual_seed(seed)


def packed(codes, scales):
    """Codes [V,d] and scales [V, groups] as the header lays them out: element by element."""
    V, d = codes.shape
    rows, blocks = -(-V // 16), -(-d // 128)
    words = np.full((rows, blocks, 256), 0x88888888, dtype=np.uint32)
    c = codes.numpy().astype(np.uint32)
    for i in range(d):
        j, g, e = i % 128 // 32, i % 32 // 8, i % 8
        bit = 4 * (e // 2) + 16 * (e % 2)
        for v in range(V):
            at = (v // 16, i // 128, 64 * g + 4 * (v % 16) + j)
            words[at] = words[at] & np.uint32(~(15 << bit) & 0xFFFFFFFF) | c[v, i] << np.uint32(bit)
    s = torch.zeros((rows * 16, scales.shape[1]), dtype=scales.dtype)
    s[:V] = scales
    return torch.from_numpy(words.view(np.uint8).reshape(rows, blocks, 1024)).cuda(), s.view(rows, 16, -1).transpose(1, 2).contiguous().cuda()


def quantized(W, group, scale_dtype):
    """The definition: (codes [V,d], scales [V, groups]).  W is float32 or 16 bits; the quotients and products below are exact in 64 bits where a tie is decided."""
    V, d = W.shape
    G = -(-d // group)
    w = torch.zeros((V, G * group), dtype=torch.float64)
    w[:, :d] = W.double()
    w = w.view(V, G, group)
    bad = ~torch.isfinite(w).all(2)
    most = torch.where(bad[..., None], torch.zeros_like(w), w).abs().amax(2)
    bits, low = (11, -24) if scale_dtype == torch.float16 else (8, -133)
    exponent = torch.frexp(most / 7)[1].clamp(min=low + bits)               # (subnormal scales have fewer bits)
    s = torch.ldexp(torch.round(torch.ldexp(most / 7, bits - exponent)), exponent - bits)
    bad |= s > torch.finfo(scale_dtype).max
    q = torch.round(w / torch.where(s > 0, s, torch.ones_like(s))[..., None]).clamp(-7, 7)
    q = torch.where(((s > 0) & ~bad)[..., None], q, torch.zeros_like(q))
    s = torch.where(bad, torch.full_like(s, float("nan")), s)
    return (q.view(V, -1)[:, :d] + 8).to(torch.uint8), s.to(scale_dtype)


def head(V, d, group, scale="bf16", seed=0, exact=False):
    g = generator(seed)
    codes = torch.randint(0, 16, (V, d), generator=g).to(torch.uint8)
    G = -(-d // group)
    if exact:                                          # powers of two: nothing is rounded
        scales = torch.pow(2.0, torch.randint(-2, 3, (V, G), generator=g).float())
    else:
        scales = 0.01 + torch.rand((V, G), generator=g)
    scales = scales.to(SCALES[scale])
    w = scales.double().repeat_interleave(group, dim=1)[:, :d] * (codes.double() - 8)
    return packed(codes, scales), w


SHAPES = [(1, 1), (5, 33), (16, 128), (37, 200), (50, 300), (33, 1001)]


@pytest.mark.parametrize("scale", ["bf16", "f16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V,d", SHAPES)
def test_quantize_is_the_definition(V, d, dtype, group, scale):
    W = (torch.randn((V, d), generator=generator(V * d)) * 0.03).to(DTYPES[dtype])
    codes, scales = quantized(W, group, SCALES[scale])
    want_codes, want_scales = packed(codes, scales)
    got_codes, got_scales = tr.head_quantize_q4(W.cuda(), group, scale_dtype=SCALES[scale])
    assert torch.equal(got_scales, want_scales) and torch.equal(got_codes, want_codes)
    back = tr.head_dequantize_q4(got_codes, got_scales, V, d, DTYPES[dtype], group)
    # 8 or 11 bits times 4 bits: exact in 32 bits, rounded once to 16
    values = (scales.float().repeat_interleave(group, dim=1)[:, :d] * (codes.float() - 8)).to(DTYPES[dtype])
    assert torch.equal(back.cpu(), values)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_quantize_ties_and_their_neighbours(dtype):
    """Weights in the middle between two codes go to the even one; fp32 weights one step beside it to the nearer."""
    s = 0.125
    grid = torch.arange(-14, 15).float() * s / 2
    W = grid.repeat(5, 1)
    if dtype == "f32":
        W[1], W[2] = torch.nextafter(grid, torch.tensor(9.0)), torch.nextafter(grid, torch.tensor(-9.0))
        W[1:3, 0], W[1:3, -1] = -7 * s, 7 * s
        W[3] *= 3.0
        W[4] = torch.nextafter(W[3], torch.tensor(0.0))
    W = W.to(DTYPES[dtype])
    codes, scales = quantized(W, 32, torch.bfloat16)
    got = tr.head_quantize_q4(W.cuda(), 32)
    assert all(torch.equal(a, b) for a, b in zip(got, packed(codes, scales)))
    assert codes[0, :5].tolist() == [1, 2, 2, 2, 3]     # -7, -6.5, -6, -5.5, -5


@pytest.mark.parametrize("scale", ["bf16", "f16"])
def test_scales_at_midpoints(scale):
    """Quotients m / 7 that are midpoints of the scale's type, and the fp32 values on both sides of 7 times one."""
    half = 2.0 ** -8 if scale == "bf16" else 2.0 ** -11
    k = torch.arange(0, 100).float() * 2 * half + 1 + half
    m = torch.cat((k * 7, torch.nextafter(k * 7, torch.tensor(99.0)), torch.nextafter(k * 7, torch.tensor(0.0)), k * 7 * 2.0 ** -20))
    W = torch.zeros((len(m), 32))
    W[:, 3] = m
    W[:, 4] = -m / 3
    codes, scales = quantized(W, 32, SCALES[scale])
    got = tr.head_quantize_q4(W.cuda(), 32, scale_dtype=SCALES[scale])
    assert all(torch.equal(a, b) for a, b in zip(got, packed(codes, scales)))


@pytest.mark.parametrize("scale", ["bf16", "f16"])
def test_quantize_of_what_is_not_ordinary(scale):
    W = torch.randn((40, 96), generator=generator(3))
    W[0] = 0
    W[1, 5], W[2, 40], W[3, 95] = float("nan"), float("inf"), float("-inf")
    W[4], W[5] = W[4] * 1e-38, W[5] * 1e-41             # scales that are subnormal or zero
    W[6] *= 2.0 ** -22                                  # subnormal fp16 scales: the codes stop at 7
    W[7] *= 1e6                                         # beyond fp16
    W[8] *= 1e38
    codes, scales = quantized(W, 32, SCALES[scale])
    got_codes, got_scales = tr.head_quantize_q4(W.cuda(), 32, scale_dtype=SCALES[scale])
    want_codes, want_scales = packed(codes, scales)
    nan = torch.isnan(want_scales)
    assert torch.equal(torch.isnan(got_scales), nan) and torch.equal(got_scales[~nan], want_scales[~nan]) and torch.equal(got_codes, want_codes)
    assert nan.sum() == (3 + (6 if scale == "f16" else 0))
    back = tr.head_dequantize_q4(got_codes, got_scales, 40, 96, torch.float32, 32).cpu()
    assert torch.isnan(back[1, :32]).all() and torch.isfinite(back[1, 32:]).all() and (back[0] == 0).all()


def test_quantize_takes_rows_with_gaps_and_offsets():
    wide = torch.randn((21, 150), generator=generator(5)).to(torch.float16).cuda()
    for a, d in ((1, 100), (8, 128), (3, 64)):
        W = wide[:, a:a + d]
        assert all(torch.equal(x, y) for x, y in zip(tr.head_quantize_q4(W, 64), tr.head_quantize_q4(W.contiguous(), 64)))


TS = (1, 2, 15, 16, 17, 33, 49, 64, 65, 97, 130, 257)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,V", [(1, 1), (31, 17), (32, 16), (129, 50), (256, 300), (1000, 70)])
def test_logits_where_nothing_is_rounded(d, V, dtype, group):
    """Rows of small integers and scales that are powers of two: the terms of a group's sum are multiples of 1/16 and their sums stay below 2^20, a row's sums are multiples of
    2^-6 below 2^18 -- at most 24 bits, so every sum is exact in 32 bits, and so are the logits.  fp32 rows of few columns: integers up to 256004, where it takes three bf16 terms
    to hold one; up to 32 of them times 1.94 and 1.5 reach 2^24.8 in steps of 1/16, 29 bits, so each of the 6 * 32 terms of the group's sum may round, by 2^-23 of 3.44 sum |x|
    at most, and s times 16 times that is the bound."""
    (codes, scales), w = head(V, d, group, exact=True, seed=d + V)
    for T in TS:
        g = generator(T)
        x = torch.randint(-4, 5, (T, d), generator=g).double()
        bound = torch.zeros((T, V), dtype=torch.float64)
        if dtype == "f32" and d <= 32:
            x += torch.randint(-1000, 1001, (T, d), generator=g) * 256.0
            bound = x.abs().sum(1, keepdim=True) * scales.cpu().double().transpose(1, 2).reshape(-1)[None, :V] * (16 * 3.44 * 6 * 32 * 2.0 ** -23)
        got = tr.head_logits_q4(x.to(DTYPES[dtype]).cuda(), codes, scales, V, group)
        off = (got.cpu().double() - x @ w.T).abs()
        assert bool((off <= bound).all()), f"T={T}: {off.max()}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,d,group", [(200003, 40, 32), (100, 2100, 128), (3000, 1300, 64)])
def test_logits_of_many_and_of_few_tokens(V, d, group, dtype):
    """More tiles of tokens than the chip takes at a time, and so few that waves share the columns of one; sums as above, of integers of one bit fewer."""
    g = generator(d)
    codes, scales = torch.randint(0, 16, (V, d), generator=g, device="cpu").to(torch.uint8), torch.pow(2.0, torch.randint(-2, 3, (V, -(-d // group)), generator=g).float())
    rows, blocks = -(-V // 16), -(-d // 128)
    full = torch.full((rows * 16, blocks * 128), 8, dtype=torch.uint8)
    full[:V, :d] = codes
    n = full.view(rows, 16, blocks, 4, 4, 4, 2).permute(0, 2, 4, 1, 3, 6, 5).reshape(rows, blocks, 1024, 2)
    s = torch.zeros((rows * 16, scales.shape[1]))
    s[:V] = scales
    s = s.view(rows, 16, -1).transpose(1, 2).contiguous().to(torch.bfloat16).cuda()
    packed_codes = (n[..., 0] | n[..., 1] << 4).contiguous().cuda()
    w = scales.double().repeat_interleave(group, dim=1)[:, :d] * (codes.double() - 8)
    for T in (1, 3, 9, 16, 20, 40, 100, 300):
        if T > 100 and V > 100000:
            continue
        x = torch.randint(-2, 3, (T, d), generator=generator(T)).double()
        got = tr.head_logits_q4(x.to(DTYPES[dtype]).cuda(), packed_codes, s, V, group)
        assert torch.equal(got.cpu().double(), x @ w.T), f"T={T}"


@pytest.mark.parametrize("scale", ["bf16", "f16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_logits_of_random_rows(dtype, group, scale):
    """A group's sum has 2 * group terms (fp32 rows: three times as many) of up to 1.94 |x| and 1.5 |x| and rounds at most once for each, by 2^-23 of what is added up so far;
    a group's product with its scale is added with one rounding of at most the sum of all magnitudes, 8 s |x| each."""
    V, d = 200, 777
    (codes, scales), w = head(V, d, group, scale, seed=group)
    for T in (1, 5, 40, 200):
        x = torch.randn((T, d), generator=generator(T)).to(DTYPES[dtype])
        got = tr.head_logits_q4(x.cuda(), codes, scales, V, group).cpu().double()
        s = scales.cpu().double().transpose(1, 2).reshape(-1, scales.shape[1])[:V]
        size = torch.nn.functional.pad(x.double().abs(), (0, -d % group)).view(T, -1, group).sum(2) @ s.T
        terms = 2 * group * (3 if dtype == "f32" else 1)
        bound = size * (16 * 3.44 * terms * 2.0 ** -23 + 8 * s.shape[1] * 2.0 ** -24)
        assert ((got - x.double() @ w.T).abs() <= bound).all()


@pytest.mark.parametrize("d", [32, 64, 128])
def test_fp32_rows_round_a_group_once(d):
    """x = 1024 m + r with m of 8 bits and r of 10: the first term of a row's value is 1024 m, whose sums with up to 128 codes and the offset are multiples of 2^6 below 2^27, and
    the rest's are multiples of 2^-4 below 2^18.  Both are exact in 32 bits, so one rounding is left, of their sum, which is the logit divided by a power of two."""
    V = 50
    (codes, scales), w = head(V, d, d, exact=True, seed=d)
    for T in (1, 3, 9, 16, 20, 70):
        g = generator(T + d)
        x = 1024.0 * torch.randint(128, 256, (T, d), generator=g) + torch.randint(0, 1024, (T, d), generator=g)
        got = tr.head_logits_q4(x.cuda(), codes, scales, V, d)
        assert torch.equal(got.cpu(), (x.double() @ w.T).float()), f"T={T}"


def test_a_row_or_a_token_that_is_not_finite_stays_alone():
    V, d = 70, 160
    (codes, scales), w = head(V, d, 32, exact=True)
    x = torch.randint(-4, 5, (20, d), generator=generator(1)).float()
    clean = tr.head_logits_q4(x.cuda(), codes, scales, V, 32)
    for dtype in DTYPES.values():
        y = x.clone()
        y[3, 7], y[9, 0], y[17, 159] = float("nan"), float("inf"), float("-inf")
        got = tr.head_logits_q4(y.to(dtype).cuda(), codes, scales, V, 32)
        bad = torch.zeros(20, dtype=torch.bool)
        bad[[3, 9, 17]] = True
        assert torch.isnan(got[bad.cuda()]).all() and torch.equal(got[~bad.cuda()], clean[~bad.cuda()])
    broken = scales.clone()
    broken[2, 1, 5] = float("nan")                      # token 37
    got = tr.head_logits_q4(x.cuda(), codes, broken, V, 32)
    assert torch.isnan(got[:, 37]).all()
    got[:, 37] = clean[:, 37]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_and_logits_with_strides(dtype):
    V, d = 50, 130
    (codes, scales), w = head(V, d, 64, exact=True)
    wide = torch.randint(-4, 5, (19, 300), generator=generator(2)).to(DTYPES[dtype]).cuda()
    out = torch.full((19, 80), 7.0, device="cuda")
    for a in (0, 1, 8, 13):
        got = tr.head_logits_q4(wide[:, a:a + d], codes, scales, V, 64, out=out[:, 11:11 + V])
        assert torch.equal(got.cpu().double(), wide[:, a:a + d].cpu().double() @ w.T)
    out[:, 11:11 + V] = 7.0
    assert (out == 7.0).all()
    last = wide.view(1, 19, 300)[:, -1, :d]             # one row of a long sequence
    assert torch.equal(tr.head_logits_q4(last, codes, scales, V, 64).cpu().double(), last.cpu().double() @ w.T)
    assert tr.head_logits_q4(wide[:0, :d], codes, scales, V, 64).shape == (0, V)


def test_what_lies_beyond_the_head_does_not_count():
    """Columns from d on and rows from V on of the last tiles may hold anything."""
    V, d = 21, 70
    (codes, scales), w = head(V, d, 32, exact=True)
    x = torch.randint(-4, 5, (4, d), generator=generator(4)).to(torch.bfloat16).cuda()
    want = tr.head_logits_q4(x, codes, scales, V, 32)
    row = torch.arange(codes.shape[0], device="cuda")[:, None, None] * 16 + torch.arange(1024, device="cuda").view(1, 1, 1024) // 16 % 16
    j, g = torch.arange(1024, device="cuda").view(1, 1, 1024) % 16 // 4, torch.arange(1024, device="cuda").view(1, 1, 1024) // 256
    beyond = (row >= V) | (32 * j + 8 * g >= 72)        # (whole words)
    codes = torch.where(beyond, torch.full_like(codes, 0xFF), codes)
    scales = scales.clone()
    scales[1, :, 5:] = float("nan")
    assert torch.equal(tr.head_logits_q4(x, codes, scales, V, 32), want)


def test_another_stream_and_a_replayed_graph():
    V, d, T = 300, 256, 7
    (codes, scales), w = head(V, d, 128, exact=True)
    x = torch.randint(-4, 5, (T, d), generator=generator(1)).to(torch.bfloat16).cuda()
    out, space = torch.empty((T, V), device="cuda"), torch.empty(tr.head_logits_q4_bytes(tr.BF16, 64, d, V), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tr.head_logits_q4(x, codes, scales, V, 128, out=out, workspace=space)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            tr.head_logits_q4(x, codes, scales, V, 128, out=out, workspace=space)
    for seed in range(4):
        x.copy_(torch.randint(-4, 5, (T, d), generator=generator(10 + seed)))
        out.fill_(0.0)
        space.fill_(255)                                # it keeps nothing
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, tr.head_logits_q4(x, codes, scales, V, 128)) and torch.equal(out.cpu().double(), x.cpu().double() @ w.T)
