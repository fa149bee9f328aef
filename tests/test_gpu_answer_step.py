"""The answer operators run together, as a decode step at the exits runs them: exits, rows, logits under a head in four bits, the rules, the token."""
import pytest
import torch

from test_gpu_logit_rules import picked, ruled

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    tide_route.load_library()
    return tide_route


def inputs(dtype, T, seed=0, C=3, d=256, V=3001, group=64):
    from paper_2603_21365_amd import exit_answer as ea, tide_route as tr
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    hidden, final = randn(C, T, d).to(dtype), randn(T, d).to(dtype)
    codes = {torch.float32: tr.F32, torch.float16: tr.F16, torch.bfloat16: tr.BF16}
    routers = ea.Routers(tr.router_pack(codes[dtype], None, randn(C, d, 128) * d ** -0.5), 1e-6, None, randn(C, 128), 0.0, 0.5, [3, 7, 11], 0, 16)
    head = ea.Head.of((randn(V, d) * (2.0 / d ** 0.5)).to(dtype), group)
    gain = 1.0 + 0.1 * randn(d)
    past = torch.randint(-1, V, (T, 40), generator=g, device="cuda", dtype=torch.int32)
    rules = {"past": past, "past_len": torch.randint(0, 41, (T,), generator=g, device="cuda", dtype=torch.int32), "repetition": torch.full((T,), 1.3, device="cuda"),
             "presence": torch.full((T,), 0.2, device="cuda"), "frequency": torch.full((T,), 0.1, device="cuda"),
             "bias_ids": past[:, :5].contiguous(), "bias_values": randn(T, 5),
             "allowed": torch.randint(-2 ** 31, 2 ** 31 - 1, (T, (V + 31) // 32), generator=g, device="cuda", dtype=torch.int32)}
    return hidden, final, routers, gain, head, rules


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T", [1, 5, 33])
def test_a_step_is_its_parts(tr, name, T):
    """Exits and rows are those of the operators that are tested elsewhere; from the rows on everything is done again in 64 bits.  A logit has less than 2 * 64 + 4 terms' roundings of
    2^-23 (three times the terms in fp32) of 16 * 3.44 times sum |x| s, and rules of at most six operations, which stretch a difference by at most the repetition's 1.3; tokens agree where the
    best is ahead of the second by what both may be off."""
    from paper_2603_21365_amd import exit_answer as ea
    hidden, final, routers, gain, head, rules = inputs(DTYPES[name], T, seed=T)
    got = ea.answer_step(hidden, final, routers, gain, 1e-6, head, **rules)
    d = hidden.shape[-1]
    exits, _, _ = tr.select_exit_packed(hidden, routers.packed, routers.eps, None, routers.w2, 0.0, 0.5, routers.layer_ids, 0, 16, d=d)
    assert torch.equal(got.exit_layer, exits) and len(set(exits.tolist())) > (T > 5)
    rows = tr.exit_project(hidden, final, exits, routers.layer_ids, gain, 1e-6)
    W = tr.head_dequantize_q4(head.codes, head.scales, head.V, d, torch.float32, head.group)
    z = rows.double().cpu() @ W.double().cpu().T
    s = head.scales.double().cpu().transpose(1, 2).reshape(-1, head.scales.shape[1])[:head.V]
    terms = 2 * head.group * (3 if name == "f32" else 1)
    off = rows.double().abs().cpu().view(T, -1, head.group).sum(2) @ s.T * (16 * 3.44 * terms * 2.0 ** -23) + 2.0 ** -21 * (z.abs() + 20)
    want = ruled({**{k: v.cpu() for k, v in rules.items()}, "logits": z.float()})
    token, log_prob = picked(want)
    for t in range(T):
        order = want[t].argsort()[::-1][:2]
        if want[t][order[0]] - want[t][order[1]] > 1.3 * float(off[t, order.tolist()].sum()):
            assert int(got.token[t]) == token[t]
        # the sum of exponentials moves by at most the largest shift of a logit, and so does the token's own
        assert abs(float(got.log_prob[t]) - log_prob[t]) <= 2.6 * float(off[t].max()) + 1e-4


def test_steps_in_a_replayed_graph(tr):
    from paper_2603_21365_amd import exit_answer as ea
    hidden, final, routers, gain, head, rules = inputs(torch.bfloat16, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ea.answer_step(hidden, final, routers, gain, 1e-6, head, **rules)      # the routers' workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = ea.answer_step(hidden, final, routers, gain, 1e-6, head, **rules)
        side.synchronize()
        for seed in range(1, 5):
            new_hidden, new_final, _, _, _, new_rules = inputs(torch.bfloat16, 4, seed=seed)
            hidden.copy_(new_hidden), final.copy_(new_final)
            for k, v in rules.items():
                v.copy_(new_rules[k])
            graph.replay()
            side.synchronize()
            got = (out.token.clone(), out.log_prob.clone(), out.exit_layer.clone())
            want = ea.answer_step(hidden, final, routers, gain, 1e-6, head, **rules)
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, (want.token, want.log_prob, want.exit_layer)))


def test_the_example_runs(tr):
    from paper_2603_21365_amd import exit_answer
    tokens = exit_answer.main(steps=3)
    assert len(tokens) == 3 and all(0 <= t < 8000 for row in tokens for t in row)
