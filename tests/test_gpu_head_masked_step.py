"""Rows without a gradient through the whole step at the exits: what they hold -- NaN, infinities -- reaches neither the head's nor the gain's gradient."""
import pytest

from test_gpu_head import types

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    import torch
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    tide_route.load_library()
    return tide_route


def states(dtype, C, T, d, seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    exits = (4 * torch.randint(0, C + 1, (T,), generator=g, device="cuda") + 3).to(torch.int32)
    return rand(C, T, d).to(dtype), rand(T, d).to(dtype), exits, [4 * c + 3 for c in range(C)], 1 + 0.1 * rand(d), rand(T, d).to(dtype), g


# every form of the kernel: a wave per row, a workgroup, and rows of 5 to 16 chunks a thread
@pytest.mark.parametrize("name,C,T,d", [("bf16", 3, 40, 768), ("f16", 2, 1300, 64), ("bf16", 2, 900, 4096), ("f32", 2, 30, 2048), ("bf16", 2, 20, 16384), ("f32", 2, 12, 16384), ("f32", 2, 1, 1600)])
@pytest.mark.parametrize("eps", [1e-6, 0.0])
def test_projection_gradient_of_rows_without_an_upstream_gradient(tr, name, C, T, d, eps):
    import torch
    hidden, final, exits, ids, gain, dy, _ = states(types()[name], C, T, d, T + d)
    none = torch.arange(T, device="cuda") % 3 == 0
    dy[none] = 0
    dy[1::6] *= -1
    clean = [t.clone() for t in (hidden, final)]
    for c, t in enumerate((*hidden, final)):
        t[0::6, c % d] = float("nan")
        t[3::6, (c + 5) % d] = float("inf")
    print(f"[gpu-case] masked projection {name} T={T} d={d} eps={eps}", flush=True)
    want, want_gain = tr.exit_project_grad(*clean, exits, ids, gain, eps, dy)
    got, got_gain = tr.exit_project_grad(hidden, final, exits, ids, gain, eps, dy)
    torch.cuda.synchronize()
    assert (got[none] == 0).all() and torch.equal(got[~none], want[~none]) and torch.equal(got_gain, want_gain) and want_gain.isfinite().all()
    if T > 1:                                          # a row with an upstream gradient is not hidden
        dy[0, 0] = 1.0
        got, got_gain = tr.exit_project_grad(hidden, final, exits, ids, gain, eps, dy)
        assert got[0].isnan().any() and got_gain.isnan().any()


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("T", [50, 300])
def test_a_step_with_broken_rows_that_have_no_target(tr, name, T):
    import torch
    from paper_2603_21365_amd.exit_tuning import exit_step
    C, d, V = 2, 128, 600
    hidden, final, exits, ids, gain, _, g = states(types()[name], C, T, d, 2)
    head = (torch.randn(V, d, generator=g, device="cuda") * 0.1).to(types()[name])
    target = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    target[::5] = -1
    print(f"[gpu-case] masked step {name} T={T}", flush=True)
    want = exit_step(hidden, final, exits, ids, gain, 1e-6, head, target=target)
    hidden[:, ::10], final[::10] = float("nan"), float("nan")
    hidden[:, 5::10], final[5::10] = float("inf"), float("inf")
    got = exit_step(hidden, final, exits, ids, gain, 1e-6, head, target=target)
    for a, b in zip(vars(got).values(), vars(want).values()):
        assert b.isfinite().all() and torch.equal(a, b)
