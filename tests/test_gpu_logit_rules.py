"""The rules of decoding on the GPU, against the definition in 64 bits and, where every operation is rounded by itself, against the same operations in 32 bits."""
import numpy as np
import pytest
import torch

from paper_2603_21365_amd import tide_route as tr

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def case(T, V, H=0, B=0, *, mask=None, dtype="f32", seed=0, lengths=True, spread=None):
    """Arguments of a call, on the CPU.  ``spread``: past and biases fall on that many tokens."""
    g = torch.Generator().manual_seed(seed * 7919 + T * 31 + V)
    rand = lambda *s: torch.rand(s, generator=g)
    tokens = lambda *s: (rand(*s) * (spread or V)).int().clamp(max=V - 1)
    c = {"logits": (torch.randn((T, V), generator=g) * 3).to(DTYPES[dtype])}
    if H:
        past = tokens(T, H)
        c["past"] = torch.where(rand(T, H) < 0.05, torch.tensor(-1, dtype=torch.int32), torch.where(rand(T, H) < 0.02, torch.tensor(V, dtype=torch.int32), past))
        if lengths:
            c["past_len"] = (rand(T) * (H + 1)).int()
            c["prompt_len"] = (c["past_len"] * rand(T)).int()
        c["repetition"], c["presence"], c["frequency"] = 0.7 + rand(T), rand(T), rand(T)
    if B:
        c["bias_ids"] = torch.where(rand(T, B) < 0.1, torch.tensor(-1, dtype=torch.int32), tokens(T, B))
        c["bias_values"] = torch.randn((T, B), generator=g) * 2
    if mask is not None:
        bits = rand(T, (V + 31) // 32, 32) < mask
        words = (bits.long() << torch.arange(32)).sum(2)
        c["allowed"] = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
    return c


def ruled(c, kind=np.float64):
    """The rules token by token; kind np.float32: each operation rounded to 32 bits."""
    z = c["logits"].float().numpy().astype(kind)
    T, V = z.shape
    f = lambda name, t: kind(c[name][t].item()) if name in c else kind(1.0 if name == "repetition" else 0.0)
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(T):
            if "past" in c:
                n = int(c["past_len"][t]) if "past_len" in c else c["past"].shape[1]
                start = int(c["prompt_len"][t]) if "prompt_len" in c else 0
                past = c["past"][t, :max(n, 0)].tolist()
                own = past[max(start, 0):]
                for v in sorted(set(past)):
                    if 0 <= v < V:
                        z[t, v] = z[t, v] / f("repetition", t) if z[t, v] > 0 else z[t, v] * f("repetition", t)
                for v in sorted(set(own)):
                    if 0 <= v < V:
                        z[t, v] = z[t, v] - kind(kind(f("frequency", t) * kind(own.count(v))) + f("presence", t))
            if "bias_ids" in c:
                sums = {}
                for v, b in zip(c["bias_ids"][t].tolist(), c["bias_values"][t].tolist()):
                    if 0 <= v < V:
                        sums[v] = kind(sums[v] + kind(b)) if v in sums else kind(b)
                for v, b in sums.items():
                    z[t, v] = z[t, v] + b
            if "allowed" in c:
                v = np.arange(V)
                z[t, (c["allowed"][t].numpy().view(np.uint32)[v // 32] >> (v % 32) & 1) == 0] = -np.inf
    return z


def picked(z):
    """(token, log_prob) of ruled logits."""
    token, log_prob = [], []
    for row in z.astype(np.float64):
        if np.isnan(row).any() or (row == np.inf).sum() > 1:
            token.append(-1), log_prob.append(np.nan)
        elif (row == -np.inf).all():
            token.append(-1), log_prob.append(-np.inf)
        else:
            k = int(row.argmax())
            rest = np.exp(np.delete(row, k) - row[k]) if row[k] != np.inf else np.zeros(1)
            token.append(k), log_prob.append(-np.log1p(rest.sum()))
    return np.array(token), np.array(log_prob)


def gpu(c):
    return {k: v.cuda() for k, v in c.items()}


def same(a, b):
    return a.dtype == b.dtype and torch.equal(a.view(torch.int32 if a.element_size() == 4 else torch.int16), b.view(torch.int32 if b.element_size() == 4 else torch.int16))


def check_rules(c):
    got = tr.logit_rules(**gpu(c)).cpu()
    want = torch.from_numpy(ruled(c, np.float32)).to(c["logits"].dtype)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert same(torch.where(nan, torch.zeros_like(got), got), torch.where(nan, torch.zeros_like(want), want))


def check_pick(c):
    """The token is that of the same operations in 32 bits.  log_prob: each exponential is off by the rounding of its exponent (|a| <= 150 here: 2^-24 * 150 * log2 e twice) and by
    2^-22 of itself, and the sum by 2^-24 for each of its additions -- a thread's own, then some 20 joins, at most V / 256 + 40."""
    token, log_prob = (x.cpu() for x in tr.logit_pick(**gpu(c)))
    want_token, want = picked(ruled(c, np.float32))
    assert token.tolist() == want_token.tolist()
    want = torch.from_numpy(want)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(log_prob), torch.isnan(want)) and torch.equal(log_prob[~fine & ~torch.isnan(want)].double(), want[~fine & ~torch.isnan(want)])
    rel = 2.0 ** -24 * (2 * 150 * 1.4427 + 4 + c["logits"].shape[1] / 256 + 40)
    # -log1p(r) moves by at most r / (1 + r) of r's relative error, and is rounded itself
    off = (log_prob.double() - want).abs()[fine]
    bound = (1 - torch.exp(want[fine])) * rel + want[fine].abs() * 2.0 ** -22 + 1e-37
    assert (off <= bound).all(), (off - bound).max()


SIZES = [(1, 1), (1, 31), (3, 33), (2, 1000), (5, 1023), (4, 1025), (3, 5003), (1, 50261), (300, 70)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V", SIZES)
def test_all_rules_together(T, V, dtype):
    for seed, (H, B, mask) in enumerate([(0, 0, None), (1, 1, 0.5), (40, 0, None), (0, 30, None), (0, 0, 0.3), (257, 300, 0.9)]):
        c = case(T, V, H, B, mask=mask, dtype=dtype, seed=seed)
        check_rules(c)
        check_pick(c)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_many_entries_of_few_tokens(dtype):
    """A past that repeats a handful of tokens, biases of which each token has dozens: counts and sums in order."""
    c = case(3, 3000, 700, 1024, dtype=dtype, spread=9, lengths=False)
    check_rules(c)
    check_pick(c)
    check_rules(case(2, 40, 5000, 500, mask=0.6, dtype=dtype))


def test_lengths_of_zero_and_beyond():
    c = case(6, 200, 50, seed=4)
    c["past_len"] = torch.tensor([0, -3, 50, 51, 1000, 7], dtype=torch.int32)
    c["prompt_len"] = torch.tensor([0, 0, 50, 60, -1, 9], dtype=torch.int32)
    c["past_len"], want = c["past_len"], c["past_len"].clamp(0, 50)
    got = tr.logit_rules(**gpu(c)).cpu()
    c["past_len"] = want
    assert same(got, torch.from_numpy(ruled(c, np.float32)))
    for name in ("past_len", "prompt_len", "repetition", "presence", "frequency"):
        part = {k: v for k, v in c.items() if k != name}
        check_rules(part)


def test_penalties_against_64_bits():
    """Four operations, each off by at most 2^-24 of the largest value on the way."""
    c = case(8, 4000, 3000, 200, seed=9)
    want = ruled(c)
    size = np.abs(c["logits"].numpy().astype(np.float64)) * 2 + 1.0 * 3000 + 1.0 + 60
    got = tr.logit_rules(**gpu(c)).cpu().numpy()
    assert (np.abs(got - want) <= 6 * 2.0 ** -24 * size).all()


def test_rows_that_leave_nothing_and_what_masked_places_hold():
    c = case(9, 3000, 30, 5, mask=0.5, seed=2)
    bits = c["allowed"]
    c["logits"][1, ::3], c["logits"][1, 1::7] = float("nan"), float("inf")
    word = torch.zeros((94, 32), dtype=torch.long)
    word[:, :] = 1
    word.view(-1)[0:3000:3] = 0
    word.view(-1)[1:3000:7] = 0
    packed = (word << torch.arange(32)).sum(1)
    bits[1] = torch.where(packed >= 1 << 31, packed - (1 << 32), packed).int()      # NaN and +inf are all masked
    bits[2] = 0
    bits[3] = 0
    c["logits"][3] = float("nan")
    c["logits"][4] = -float("inf")
    c["logits"][5, 700] = float("inf")
    bits[5, 700 // 32] |= 1 << (700 % 32)
    c["logits"][6, [5, 2999]] = float("nan")
    bits[6] = -1
    c["logits"][7, [5, 2999]] = float("inf")
    bits[7] = -1
    c["logits"][8] = torch.finfo(torch.float32).min
    check_rules(c)
    check_pick(c)
    token, log_prob = tr.logit_pick(**gpu(c))
    assert token.tolist()[2:5] == [-1, -1, -1] and token[5] == 700 and log_prob[5] == 0 and token.tolist()[6:8] == [-1, -1]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_lowest_of_equal_logits(dtype):
    for V in (7, 1030, 20011):
        z = torch.zeros((4, V), dtype=DTYPES[dtype])
        z[1, V - 1] = z[1, V // 2] = z[1, V // 3] = 1.0
        z[2] = -5.0
        z[3, 0] = z[3, V - 1] = 3.0
        token, log_prob = tr.logit_pick(z.cuda())
        assert token.tolist() == [0, V // 3, 0, 0]
        check_pick({"logits": z})


def test_a_certain_token_keeps_the_digits_of_its_log_probability():
    z = torch.full((2, 5000), -30.0)
    z[0, 77] = 0.0
    z[1, 4999] = 10.0
    check_pick({"logits": z})
    assert (tr.logit_pick(z.cuda())[1] < 0).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_strides_places_and_what_lies_beside(dtype):
    T, V = 5, 1001
    c = gpu(case(T, V, 20, 10, mask=0.7, dtype=dtype))
    want, (token, log_prob) = tr.logit_rules(**c), tr.logit_pick(**c)
    wide = torch.full((T, 3 * V), 9.0, dtype=DTYPES[dtype], device="cuda")
    for a in (0, 1, 5):
        wide.fill_(9.0)
        view = wide[:, a:a + V]
        view.copy_(c["logits"])
        got = tr.logit_rules(**{**c, "logits": view}, out=wide[:, 2 * V - 3:3 * V - 3])
        assert same(got.contiguous(), want) and same(view.contiguous(), c["logits"])
        assert (wide[:, :a] == 9).all() and (wide[:, a + V:2 * V - 3] == 9).all() and (wide[:, 3 * V - 3:] == 9).all()
        pick = tr.logit_pick(**{**c, "logits": view})
        assert torch.equal(pick[0], token) and torch.equal(pick[1], log_prob)
        got = tr.logit_rules(**{**c, "logits": view}, out=view)             # in place
        assert same(got.contiguous(), want) and (wide[:, :a] == 9).all() and (wide[:, a + V:2 * V - 3] == 9).all()


def test_untouched_logits_keep_their_bits():
    z = torch.tensor([[-0.0, 0.0, float("nan"), float("inf"), -float("inf"), 1e-42, -1e-42, 3.0]])
    z.view(torch.int32)[0, 2] = 0x7F812345
    ids, values = torch.tensor([[7]], dtype=torch.int32), torch.tensor([[0.5]])
    past = torch.tensor([[7]], dtype=torch.int32)
    got = tr.logit_rules(z.cuda(), past=past.cuda(), bias_ids=ids.cuda(), bias_values=values.cuda()).cpu()
    assert same(got[:, :7].contiguous(), z[:, :7].contiguous()) and got[0, 7] == 3.5


def test_an_empty_batch_and_empty_lists():
    z = torch.randn((3, 50)).cuda()
    empty_i, empty_f = torch.zeros((3, 0), dtype=torch.int32, device="cuda"), torch.zeros((3, 0), device="cuda")
    assert same(tr.logit_rules(z, past=empty_i, bias_ids=empty_i, bias_values=empty_f), z)
    assert tr.logit_rules(z[:0]).shape == (0, 50) and tr.logit_pick(z[:0])[0].shape == (0,)


def test_results_do_not_depend_on_the_batch_or_on_timing():
    c = gpu(case(64, 9000, 500, 50, mask=0.8))
    token, log_prob = tr.logit_pick(**c)
    for _ in range(3):
        again = tr.logit_pick(**c)
        assert torch.equal(again[0], token) and torch.equal(again[1], log_prob)
    one = tr.logit_pick(**{k: v[9:10].contiguous() for k, v in c.items()})
    assert one[0][0] == token[9] and abs(one[1][0] - log_prob[9]) <= 1e-4


def test_another_stream_and_replayed_graphs_on_workspaces_of_their_own():
    c = gpu(case(5, 20000, 100, 20, mask=0.8))
    side, graphs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            space = torch.empty(tr.logit_pick_bytes(5, 20000), dtype=torch.uint8, device="cuda")
            tr.logit_pick(**c, workspace=space)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                graphs.append((graph, tr.logit_pick(**c, workspace=space), tr.logit_rules(**c), space))
    for seed in range(3):
        new = case(5, 20000, 100, 20, mask=0.8, seed=20 + seed)
        for k, v in new.items():
            c[k].copy_(v)
        for graph, (token, log_prob), out, space in graphs:
            token.fill_(-7), log_prob.fill_(1.0), out.fill_(0.0), space.fill_(255)
        torch.cuda.synchronize()
        for graph, *_ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want, ruled_now = tr.logit_pick(**c), tr.logit_rules(**c)
        for _, (token, log_prob), out, _ in graphs:
            assert torch.equal(token, want[0]) and torch.equal(log_prob, want[1]) and same(out, ruled_now)
