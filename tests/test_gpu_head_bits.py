"""How many bits the gradient to the logits is held in.  In two planes of 16 bits -- up to 64 rows, and where the caller asks for it (wide) -- what is left of dx's and
dW's rounding is the results' own: the bounds are test_gpu_head.py's with u^2 |G| for G's rounding in the place of u |G|.  (With one plane a row of dx, most of which
is its target's G times that token's row of W, is off by up to twice its rounding: beyond these bounds.)"""
import pytest

from test_gpu_head import E, Exact, half_step, make, near, types

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    import torch
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    tide_route.load_library()
    return tide_route


def gradients(ex, kept, dtype):
    """dx, dW of Exact's formulas and their bounds with G in two planes."""
    import torch
    u = half_step(dtype)
    g = torch.where(kept, ex.grad * ex.tau, 0.0)[:, None]
    x = torch.where(kept[:, None], ex.x, 0.0)
    p = torch.where(kept[:, None], torch.exp(ex.z / ex.tau - ex.lse[:, None]), 0.0)
    G = g * (p - torch.where(kept[:, None], ex.teacher, 0.0))
    tol_G = u * u * G.abs() + g.abs() * (p * ex.tol_p[:, None] + 16 * E * (p + ex.teacher))
    if dtype == torch.float16:
        tol_G = tol_G + 2.0 ** -38 * g.abs().max()
    for A, tol_A, B in ((G, tol_G, ex.W), (G.T, tol_G.T, x)):
        exact = A @ B
        yield exact
        yield tol_A @ B.abs() + A.shape[1] * E * (A.abs() @ B.abs()) + 1.01 * u * exact.abs() + (2.0 ** -25 if dtype == torch.float16 else 1e-38)


@pytest.mark.parametrize("name", ["f16", "bf16"])
@pytest.mark.parametrize("T,d,V,K", [(1, 64, 300, 0), (40, 128, 700, 0), (64, 512, 300, 5), (65, 128, 700, 0), (100, 33, 511, 4), (200, 96, 1030, 0), (300, 512, 5000, 9), (520, 768, 1537, 0),
                                     (4200, 72, 40003, 0)])
def test_two_planes(tr, name, T, d, V, K):
    import torch
    dtype = types()[name]
    x, W, target, values, ids, grad = make(dtype, T, d, V, K, T + d)
    if T > 5:
        x[4] = float("nan")                            # (its upstream gradient is zero)
    clean = torch.where(x.isnan(), 0.0, x)
    print(f"[gpu-case] wide {name} T={T} d={d} V={V} K={K}", flush=True)
    if K:
        loss, lse, _ = tr.head_distill(x, W, values, ids, 2.0)
        run = lambda **kw: tr.head_distill_grad(x, W, values, ids, 2.0, lse, grad, **kw)
    else:
        loss, lse = tr.head_loss(x, W, target)
        run = lambda **kw: tr.head_loss_grad(x, W, target, lse, grad, **kw)
    dx, dW = run(wide=True)
    torch.cuda.synchronize()
    ex = Exact(clean, W, target, values, ids, 2.0 if K else 1.0, grad)
    kept = ex.live & (grad != 0)
    want_dx, tol_dx, want_dw, tol_dw = gradients(ex, kept, dtype)
    assert (dx[~kept] == 0).all()
    near("dx", dx, want_dx, tol_dx)
    near("dW", dW, want_dw, tol_dw)
    if T <= 64:                                        # what the call does there by itself
        for a, b in zip(run(), (dx, dW)):
            assert torch.equal(a, b)
    for a, b in ((run(wide=True, want_dw=False)[0], dx), (run(wide=True, want_dx=False)[1], dW)):
        assert torch.equal(a, b)


def test_fp32_has_them_anyway(tr):
    import torch
    x, W, target, _, _, grad = make(torch.float32, 90, 64, 300, 0, 4)
    print("[gpu-case] wide f32", flush=True)
    _, lse = tr.head_loss(x, W, target)
    for a, b in zip(tr.head_loss_grad(x, W, target, lse, grad), tr.head_loss_grad(x, W, target, lse, grad, wide=True)):
        assert torch.equal(a, b)
    assert tr.head_workspace_bytes(tr.F32, 90, 64, 300, gradient=True) == tr.head_workspace_bytes(tr.F32, 90, 64, 300, gradient=True, wide=True)
