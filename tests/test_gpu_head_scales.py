"""fp32 rows of very different sizes under the head operators: what one row holds reaches no other row's loss or dx, and a row that has no gradient reaches
nothing.  The bounds are test_gpu_head.py's with a row's own size in the place of the tensor's:
  z       d e sum|x W| + 2^-21 sum|x W| + d 2^-38 max|x_t| max|W|
  G       2^-22 |G| + |g| (p tol_p + 16 e (p + teacher)) + 2^-38 |g_t|
  dx      the error of G through the product, V e + 2^-22 of sum|G W|, V 2^-38 |g_t| max|W|
  dW      the same over the rows, T 2^-38 of the largest |g_t| max|x_t| among the rows that have a gradient"""
import pytest

from test_gpu_head import E, Exact, make, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    import torch
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    tide_route.load_library()
    return tide_route


class Rows:
    """The formulas in 64 bits with bounds row by row; `kept`: the rows that have a gradient."""

    def __init__(self, x, W, values, ids, target, tau, grad, kept):
        import torch
        T, d, V = *x.shape, W.shape[0]
        x, W = x.double(), W.double()
        x = torch.where(kept[:, None], x, 0.0)
        z, size = x @ W.T, x.abs() @ W.abs().T
        self.tol_z = (d * E + 2.0 ** -21) * size + d * 2.0 ** -38 * x.abs().amax(1, keepdim=True) * W.abs().max()
        self.z, self.lse = z, torch.logsumexp(z / tau, 1)
        self.tol_lse = self.tol_z.amax(1) / tau + 2.0 ** -20 * (1 + self.lse.abs())
        teacher = torch.zeros_like(z)
        if values is None:
            t = kept.nonzero()[:, 0]
            teacher[t, target[t].long()] = 1.0
        else:
            teacher.scatter_add_(1, ids.long(), torch.softmax(values.double() / tau, 1))
        g = torch.where(kept, grad.double() * tau, 0.0)[:, None]
        p = torch.exp(z / tau - self.lse[:, None])
        tol_p = 2 * (self.tol_z.amax(1) / tau + self.tol_lse)[:, None]
        G = g * (p - teacher)
        tol_G = 2.0 ** -22 * G.abs() + g.abs() * (p * tol_p + 16 * E * (p + teacher) + 2.0 ** -38)
        w = W.abs()
        self.dx = G @ W
        self.tol_dx = tol_G @ w + (V * E + 2.0 ** -22) * (G.abs() @ w) + V * 2.0 ** -38 * g.abs() * w.max() + 1.01 * E * self.dx.abs() + 1e-37
        self.dW = G.T @ x
        largest = (g.abs()[:, 0] * x.abs().amax(1)).max()
        self.tol_dW = tol_G.T @ x.abs() + (T * E + 2.0 ** -22) * (G.T.abs() @ x.abs()) + T * 2.0 ** -38 * largest + 1.01 * E * self.dW.abs() + 1e-37


@pytest.mark.parametrize("garbage", [1e8, 1e20, 3e38])
@pytest.mark.parametrize("T,d,V", [(40, 64, 500), (128, 66, 300), (200, 128, 900), (700, 2052, 400)])
def test_rows_without_a_gradient_may_hold_anything(tr, T, d, V, garbage):
    """Finite garbage in rows without a target, and in rows whose upstream gradient is zero."""
    import torch
    x, W, target, _, _, grad = make(torch.float32, T, d, V, 0, T + d)
    clean = x.clone()
    x[1], x[T - 1], x[4] = garbage, -garbage, garbage                          # (4: a target, but no upstream gradient)
    clean[1], clean[T - 1], clean[4] = 0.0, 0.0, 0.0
    print(f"[gpu-case] garbage {garbage} T={T} d={d} V={V}", flush=True)
    loss, lse = tr.head_loss(x, W, target)
    dx, dW = tr.head_loss_grad(x, W, target, lse, grad)
    torch.cuda.synchronize()
    ex = Exact(clean, W, target, None, None, 1.0, grad)
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[1] = rows[T - 1] = rows[4] = False
    assert loss[1] == 0 and loss[T - 1] == 0
    near("lse", lse[rows], ex.lse[rows], ex.tol_lse[rows])
    near("loss", loss[rows], ex.loss[rows], ex.tol_loss[rows])
    kept = ex.live & (grad != 0)
    want_dx, tol_dx, want_dw, tol_dw = ex.gradients(kept)
    assert (dx[~kept] == 0).all()
    near("dx", dx, want_dx, tol_dx)
    near("dW", dW, want_dw, tol_dw)


@pytest.mark.parametrize("T,d,V,K,tau", [(20, 64, 300, 4, 1.0), (150, 128, 700, 8, 2.0), (260, 33, 300, 0, 1.0), (300, 2304, 600, 16, 1.0)])
def test_rows_and_gradients_of_all_sizes(tr, T, d, V, K, tau):
    """Rows from 2^-60 to 8 and upstream gradients from 2^-50 to 2^50: logits and dx are as exact in each of them."""
    import torch
    x, W, _, _, _, _ = make(torch.float32, T, d, V, 0, T + V)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")
    x = x * torch.exp2(-60 * rand(T, 1))
    x[0], x[T // 2] = 8 * torch.randn(d, generator=g, device="cuda"), 0.0
    grad = torch.exp2(100 * rand(T) - 50) * torch.where(rand(T) < 0.5, -1.0, 1.0)
    target = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    kept = torch.ones(T, dtype=torch.bool, device="cuda")
    print(f"[gpu-case] sizes T={T} d={d} V={V} K={K}", flush=True)
    if K:
        ids = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(T)]).to(torch.int32)
        values = 3 * torch.randn(T, K, generator=g, device="cuda")
        loss, lse, z = tr.head_distill(x, W, values, ids, tau)
        dx, dW = tr.head_distill_grad(x, W, values, ids, tau, lse, grad)
        want = Rows(x, W, values, ids, None, tau, grad, kept)
        near("z", z, want.z.gather(1, ids.long()), want.tol_z.gather(1, ids.long()) + 1e-37)
    else:
        loss, lse = tr.head_loss(x, W, target)
        dx, dW = tr.head_loss_grad(x, W, target, lse, grad)
        want = Rows(x, W, None, None, target, tau, grad, kept)
    near("lse", lse, want.lse, want.tol_lse)
    near("dx", dx, want.dx, want.tol_dx)
    near("dW", dW, want.dW, want.tol_dW)


# An fp32 operand's two halves: 2^-22 of the value, 2^-51 of the largest where that is more; of a product, what is dropped included, 2^-21 of it and 2^-49 of the
# largest magnitudes' product.
FLOOR = 2.0 ** -49


@pytest.mark.parametrize("T,d,V", [(150, 96, 600), (300, 520, 300)])
def test_rows_of_a_head_of_all_sizes(tr, T, d, V):
    """Logits of the head's rows from 1 down to 2^-26 of the largest are as exact, each for itself."""
    import torch
    x, W, _, _, _, _ = make(torch.float32, T, d, V, 0, V)
    W = (W * torch.exp2(-26 * torch.arange(V, device="cuda") / V)[:, None]).contiguous()
    K = 300
    ids = (torch.arange(K, device="cuda") * (V // K)).to(torch.int32).repeat(T, 1).contiguous()
    values = torch.zeros(T, K, device="cuda")
    print(f"[gpu-case] head sizes T={T} d={d} V={V}", flush=True)
    _, _, z = tr.head_distill(x, W, values, ids, 1.0)
    want, size = x.double() @ W.double().T, x.double().abs() @ W.double().abs().T
    tol = (d * E + 2.0 ** -21) * size + d * FLOOR * x.double().abs().amax(1, keepdim=True) * W.double().abs().max()
    near("z", z, want.gather(1, ids.long()), tol.gather(1, ids.long()))


@pytest.mark.parametrize("T,d,V", [(20, 64, 400), (150, 64, 400), (400, 160, 999)])
def test_improbable_tokens_keep_their_digits(tr, T, d, V):
    """Tokens down to p = e^-24 in every row: their rows of dW hold what p holds, not 2^-39 of the largest gradient."""
    import torch
    x, W, _, _, _, grad = make(torch.float32, T, d, V, 0, d)
    W = 0.2 * W
    x[:, 0] = 8.0
    W[:, 0] = -torch.arange(V, device="cuda") * (24.0 / 8 / V)
    target = torch.zeros(T, dtype=torch.int32, device="cuda")
    print(f"[gpu-case] improbable T={T} d={d} V={V}", flush=True)
    _, lse = tr.head_loss(x, W, target)
    _, dW = tr.head_loss_grad(x, W, target, lse, grad)
    X, H, g = x.double(), W.double(), grad.double()[:, None]
    z = X @ H.T
    tol_z = (d * E + 2.0 ** -21) * (X.abs() @ H.abs().T) + d * FLOOR * X.abs().max() * H.abs().max()
    exact_lse = torch.logsumexp(z, 1)
    p = torch.exp(z - exact_lse[:, None])
    assert p.min() < 2.0 ** -33
    tol_p = (tol_z + tol_z.amax(1, keepdim=True) + 2 * 2.0 ** -20 * (1 + exact_lse.abs()[:, None]))      # z's error, lse's, and the exponential's
    G = g * p
    G[:, 0] -= g[:, 0]
    tol_G = 2.0 ** -22 * G.abs() + g.abs() * (p * tol_p + 16 * E * p + FLOOR)
    tol_G[:, 0] += 16 * E * g[:, 0].abs()
    want = G.T @ X
    tol = tol_G.T @ X.abs() + (T * E + 2.0 ** -21) * (G.T.abs() @ X.abs()) + T * FLOOR * (g.abs()[:, 0] * X.abs().amax(1)).max() + 1.01 * E * want.abs()
    near("dW", dW, want, tol)
    share = ((dW.double() - want).norm(dim=1) / want.norm(dim=1)).max().item()
    print(f"HEAD largest error of a token's row of dW: {share:.2e}", flush=True)


@pytest.mark.parametrize("name", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T", [40, 200])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_a_gradient_that_is_not_finite_takes_no_other_rows_bits(tr, name, T, bad):
    """The other rows' dx is bit for bit what it is without that row."""
    import torch
    from test_gpu_head import types
    x, W, target, _, _, grad = make(types()[name], T, 64, 300, 0, 17)
    grad = grad * 2.0 ** -18
    grad[3] = 0.0
    print(f"[gpu-case] gradient {bad} {name} T={T}", flush=True)
    loss, lse = tr.head_loss(x, W, target)
    want, _ = tr.head_loss_grad(x, W, target, lse, grad)
    grad[3] = float(bad)
    got, _ = tr.head_loss_grad(x, W, target, lse, grad)
    others = torch.arange(T, device="cuda") != 3
    assert (want[others] != 0).any() and torch.equal(got[others], want[others])
    assert not got[3].isfinite().any()
