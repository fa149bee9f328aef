"""Head operators at sizes where a workgroup goes through several tiles, a whole training step at the exits, and what a call refuses on the GPU.
The tolerances are those of test_gpu_head.py; a step's gradients are held against autograd in 64 bits through the rounded rows."""
import pytest

from test_gpu_head import Exact, half_step, make, near, types

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    import torch
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    tide_route.load_library()
    return tide_route


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,d,V", [(70, 600, 40003), (2100, 8200, 900)])      # dW: 471 tiles; dx: 297 tiles
def test_more_tiles_than_workgroups(tr, name, T, d, V):
    import torch
    x, W, target, _, _, grad = make(types()[name], T, d, V, 0, 31)
    print(f"[gpu-case] tiles {name} T={T} d={d} V={V}", flush=True)
    loss, lse = tr.head_loss(x, W, target)
    dx, dW = tr.head_loss_grad(x, W, target, lse, grad)
    torch.cuda.synchronize()
    ex = Exact(x, W, target, None, None, 1.0, grad)
    near("loss", loss, ex.loss, ex.tol_loss)
    want_dx, tol_dx, want_dw, tol_dw = ex.gradients(ex.live & (grad != 0))
    near("dx", dx, want_dx, tol_dx)
    near("dW", dW, want_dw, tol_dw)


def test_small_workspace_and_wrong_types_are_refused(tr):
    import torch
    x, W, target, values, ids, grad = make(torch.bfloat16, 20, 64, 300, 4, 1)
    ws = torch.empty(tr.head_workspace_bytes(tr.BF16, 20, 64, 300) - 1, dtype=torch.uint8, device="cuda")
    print("[gpu-case] refusals", flush=True)
    with pytest.raises(tr.TideError, match="workspace"):
        tr.head_loss(x, W, target, workspace=ws)
    big = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    with pytest.raises(tr.TideError, match="aligned"):
        tr.head_loss(x, W, target, workspace=big[8:])
    for bad in (lambda: tr.head_loss(x, W.float(), target), lambda: tr.head_loss(x, W[:, :32], target), lambda: tr.head_loss(x, W, target.long()),
                lambda: tr.head_loss_grad(x, W, target, grad.double(), grad), lambda: tr.head_distill(x, W, values[:, :2], ids, 1.0),
                lambda: tr.head_loss(x, W, target[:5]), lambda: tr.head_loss(x.cpu(), W, target)):
        with pytest.raises(ValueError):
            bad()


def test_projection_gradient_on_strided_states_and_its_refusals(tr):
    import torch
    C, T, d = 2, 50, 256
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    hidden, final, dy = r(C, T, d), r(T, d), r(T, d)
    exits = (4 * torch.randint(0, C + 1, (T,), generator=g, device="cuda") + 3).to(torch.int32)
    want = tr.exit_project_grad(hidden, final, exits, [3, 7], None, 1e-6, dy)
    H = torch.full((C, T + 2, d + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    F = torch.full((T, d + 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    D = torch.full((T, d + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    H[:, :T, :d], F[:, :d], D[:, :d] = hidden, final, dy
    print("[gpu-case] strided projection gradient", flush=True)
    got = tr.exit_project_grad(H[:, :T], F, exits, [3, 7], None, 1e-6, D[:, :d])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    none = tr.exit_project_grad(hidden[:, :0], final[:0], exits[:0], [3, 7], None, 1e-6, dy[:0])
    assert none[0].shape == (0, d) and (none[1] == 0).all()
    with pytest.raises(ValueError):
        tr.exit_project_grad(hidden, final.float(), exits, [3, 7], None, 1e-6, dy)
    with pytest.raises(ValueError):
        tr.exit_project_grad(hidden, final, exits.long(), [3, 7], None, 1e-6, dy)
    with pytest.raises(tr.TideError, match="workspace"):
        tr.exit_project_grad(hidden, final, exits, [3, 7], None, 1e-6, dy, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("taught_by", ["targets", "teacher"])
def test_a_step_at_the_exits_against_autograd(tr, taught_by):
    """fp32, so that the roundings between the operators stay far below the bound: 2^-16 of the gradients' largest element (each of the chain's four sums of a few
    hundred terms is within 2^-20)."""
    import torch
    from paper_2603_21365_amd.exit_tuning import exit_step
    C, T, d, V, K, tau, eps = 3, 90, 64, 500, 5, 2.0, 1e-5
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    hidden, final, head, gain = r(C, T, d), r(T, d), r(V, d) * 0.15, 1 + 0.1 * r(d)
    exits = (4 * torch.randint(0, C + 1, (T,), generator=g, device="cuda") + 3).to(torch.int32)
    ids = [3, 7, 11]
    target = torch.randint(-50, V, (T,), generator=g, device="cuda", dtype=torch.int32).clamp(min=-1)
    top = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(T)]).to(torch.int32)
    top[3] = -1
    values = 3 * r(T, K)
    print(f"[gpu-case] step {taught_by}", flush=True)
    if taught_by == "targets":
        s = exit_step(hidden, final, exits, ids, gain, eps, head, target=target)
    else:
        s = exit_step(hidden, final, exits, ids, gain, eps, head, teacher=(values, top), tau=tau)
    torch.cuda.synchronize()
    at = (exits.long() - 3) // 4
    src = torch.cat((hidden, final[None]))[at, torch.arange(T, device="cuda")].double().requires_grad_()
    gd, W = gain.double().requires_grad_(), head.double().requires_grad_()
    z = (src * torch.rsqrt((src * src).mean(1, keepdim=True) + eps) * gd) @ W.T
    if taught_by == "targets":
        want = torch.nn.functional.cross_entropy(z, target.long(), ignore_index=-1, reduction="sum") / (target >= 0).sum()
    else:
        there = top >= 0
        q = torch.nan_to_num(torch.softmax((values.double() / tau).masked_fill(~there, -float("inf")), 1))
        logp = torch.log_softmax(z / tau, 1).gather(1, top.clamp(min=0).long())
        want = tau * tau * (torch.where(q > 0, q * torch.log(q.clamp(min=1e-300)), 0.0) - q * logp).sum() / there.any(1).sum()
    want.backward()
    assert abs(s.mean.item() - want.item()) < 2.0 ** -18 * abs(want.item())
    for name, got, w in (("rows", s.grad_rows, src.grad), ("gain", s.grad_gain, gd.grad), ("head", s.grad_head, W.grad)):
        off = (got.double() - w).abs().max().item()
        print(f"HEAD step {name}: {off / w.abs().max().item():.2e}", flush=True)
        assert off < 2.0 ** -16 * w.abs().max().item(), name


def test_tuning_lowers_the_loss(tr):
    from paper_2603_21365_amd import exit_tuning
    print("[gpu-case] tuning", flush=True)
    losses = exit_tuning.main()
    print("HEAD losses", losses, flush=True)
    assert all(b < a for a, b in zip(losses, losses[1:])) and losses[-1] < 0.9 * losses[0]


def test_loss_of_a_few_fp32_rows_is_the_planes_loss(tr):
    """The form for few fp32 rows and the planes' form agree within their bounds on the same rows."""
    import torch
    x, W, target, _, _, grad = make(torch.float32, 129, 256, 3000, 0, 2)
    print("[gpu-case] fp32 forms", flush=True)
    many, lse_many = tr.head_loss(x, W, target)
    few, lse_few = tr.head_loss(x[:128], W, target[:128].contiguous())
    ex = Exact(x, W, target, None, None, 1.0, grad)
    near("lse of few", lse_few, ex.lse[:128], ex.tol_lse[:128])
    near("lse of many", lse_many, ex.lse, ex.tol_lse)
    assert half_step(torch.float32) < ex.tol_lse.max()
