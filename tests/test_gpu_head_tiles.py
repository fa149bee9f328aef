"""Head operators on each height of tile, with hard targets and with a teacher, through several pieces of the vocabulary, on heads and rows beyond 2 GiB, and what the
fp32 planes' passes add.  A vocabulary of 33000 and more keeps the large tiles: of small ones the rows go in tiles of 64 whatever their number."""
import pytest

from test_gpu_head import E, Exact, make, near, types

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    import torch
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    tide_route.load_library()
    return tide_route


def loss_and_gradients(tr, name, T, d, V):
    import torch
    x, W, target, _, _, grad = make(types()[name], T, d, V, 0, T + d + V)
    loss, lse = tr.head_loss(x, W, target)
    dx, dW = tr.head_loss_grad(x, W, target, lse, grad)
    torch.cuda.synchronize()
    ex = Exact(x, W, target, None, None, 1.0, grad)
    near("lse", lse, ex.lse, ex.tol_lse)
    near("loss", loss, ex.loss, ex.tol_loss)
    want_dx, tol_dx, want_dw, tol_dw = ex.gradients(ex.live & (grad != 0))
    near("dx", dx, want_dx, tol_dx)
    near("dW", dW, want_dw, tol_dw)


def distillation_and_gradients(tr, name, T, d, V, K, tau, last=0):
    """last: that many of a row's tokens are among the last 300 of the vocabulary."""
    import torch
    x, W, _, values, ids, grad = make(types()[name], T, d, V, K, T + d + V + K)
    if last:
        ids[5:, :last] = V - 1 - ids[5:, :last] % 300
    loss, lse, z = tr.head_distill(x, W, values, ids, tau)
    dx, dW = tr.head_distill_grad(x, W, values, ids, tau, lse, grad)
    torch.cuda.synchronize()
    ex = Exact(x, W, None, values, ids, tau, grad)
    near("lse", lse, ex.lse, ex.tol_lse)
    near("z", z, ex.z_top, ex.tol_top + 1e-300)
    near("loss", loss, ex.loss, ex.tol_loss)
    kept = ex.live & (grad != 0)
    want_dx, tol_dx, want_dw, tol_dw = ex.gradients(kept)
    assert (dx[~kept] == 0).all()
    near("dx", dx, want_dx, tol_dx)
    near("dW", dW, want_dw, tol_dw)


# rows: tiles of 128 (one, ragged), 192 (one and two, ragged), 256 (one and three, ragged); columns: 130 tiles, the last one ragged
HEIGHTS = [(100, 64, 33001), (130, 72, 33001), (322, 64, 33001), (250, 40, 33025), (640, 64, 33001)]


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,d,V", HEIGHTS)
def test_heights_of_tiles(tr, name, T, d, V):
    print(f"[gpu-case] height {name} T={T} d={d} V={V}", flush=True)
    loss_and_gradients(tr, name, T, d, V)


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K", [2, 33])
@pytest.mark.parametrize("T,d,V", HEIGHTS)
def test_heights_of_tiles_with_a_teacher(tr, name, T, d, V, K):
    print(f"[gpu-case] height with teacher {name} T={T} d={d} V={V} K={K}", flush=True)
    distillation_and_gradients(tr, name, T, d, V, K, 2.0)


@pytest.mark.parametrize("name,T,d,V", [("f32", 3000, 64, 40001), ("f16", 4300, 64, 40001), ("bf16", 4300, 72, 40001)])
def test_a_teacher_over_several_pieces_of_the_vocabulary(tr, name, T, d, V):
    """G of more than 256 MiB: two pieces; half of each row's tokens lie at the end of the last one."""
    assert T * V * (4 if name == "f32" else 2) > 1 << 28
    print(f"[gpu-case] teacher over pieces {name} T={T} V={V}", flush=True)
    distillation_and_gradients(tr, name, T, d, V, 6, 2.0, last=3)


def test_a_head_beyond_2_gib(tr):
    """bf16, 140000 x 8192: the logits, the gradients' rows of the last tokens and dx are those of the whole head."""
    import torch
    T, d, V, K = 5, 8192, 140000, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    W = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    for a in range(0, V, 20000):
        W[a:a + 20000] = torch.randn(20000, d, generator=g, device="cuda") * (1.5 / d ** 0.5)
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    ids = (V - 1 - torch.arange(T * K, device="cuda") * 7).view(T, K).to(torch.int32)
    values, grad = torch.randn(T, K, generator=g, device="cuda"), 0.5 + torch.rand(T, generator=g, device="cuda")
    print("[gpu-case] head beyond 2 GiB", flush=True)
    loss, lse, z = tr.head_distill(x, W, values, ids, 1.0)
    dx, dW = tr.head_distill_grad(x, W, values, ids, 1.0, lse, grad)
    torch.cuda.synchronize()
    X, q = x.double(), torch.softmax(values.double(), 1)
    logits = torch.cat([X @ W[a:a + 20000].double().T for a in range(0, V, 20000)], 1)
    size = torch.cat([X.abs() @ W[a:a + 20000].double().abs().T for a in range(0, V, 20000)], 1)
    tol_z, exact_lse = d * E * size, torch.logsumexp(logits, 1)
    tol_lse = tol_z.amax(1) + 2.0 ** -20 * (1 + exact_lse)
    near("z", z, logits.gather(1, ids.long()), tol_z.gather(1, ids.long()))
    near("lse", lse, exact_lse, tol_lse)
    p = torch.exp(logits - exact_lse[:, None])
    teacher = torch.zeros_like(p).scatter_add_(1, ids.long(), q)
    G = grad.double()[:, None] * (p - teacher)
    u = 2.0 ** -8
    tol_G = u * u * G.abs() + grad.double()[:, None] * (p * 2 * (tol_z.amax(1) + tol_lse)[:, None] + 16 * E * (p + teacher))
    want, tol = torch.zeros(T, d, dtype=torch.float64, device="cuda"), torch.zeros(T, d, dtype=torch.float64, device="cuda")
    for a in range(0, V, 20000):
        w = W[a:a + 20000].double()
        want += G[:, a:a + 20000] @ w
        tol += (tol_G[:, a:a + 20000] + V * E * G[:, a:a + 20000].abs()) @ w.abs()
    near("dx", dx, want, tol + 1.01 * u * want.abs())
    for rows in (slice(0, 300), slice(131000, 131300), slice(V - 300, V)):      # 2 GiB end at row 131072
        want = G[:, rows].T @ X
        near("dW", dW[rows], want, tol_G[:, rows].T @ X.abs() + 2 * T * E * (G[:, rows].T.abs() @ X.abs()) + 1.01 * u * want.abs())


@pytest.mark.parametrize("name,T,V", [("bf16", 300, 70), ("bf16", 20, 290), ("f32", 140, 60), ("f32", 100, 150)])
def test_rows_the_largest_stride_apart(tr, name, T, V):
    """4194304 elements between the rows of x or of W: a tile's rows reach over almost 2 GiB."""
    import torch
    d, far, dtype = 64, 1 << 22, types()[name]
    x, W, target, _, _, grad = make(dtype, T, d, V, 0, T)
    n, few = max(T, V), (x if T > V else W)
    wide = torch.empty((n - 1) * far + d, dtype=dtype, device="cuda").as_strided((n, d), (far, 1))
    wide.copy_(few)
    X, H = (wide, W) if T > V else (x, wide)
    print(f"[gpu-case] far rows {name} T={T} V={V}", flush=True)
    want = tr.head_loss(x, W, target)
    got = tr.head_loss(X, H, target)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]) and want[0].isfinite().all()
    for a, b in zip(tr.head_loss_grad(x, W, target, want[1], grad), tr.head_loss_grad(X, H, target, want[1], grad)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("low_in", ["x", "W"])
@pytest.mark.parametrize("T,d,V", [(20, 1024, 300), (200, 1024, 300), (400, 512, 33001)])
def test_fp32_logits_of_whole_numbers_are_exact(tr, T, d, V, low_in):
    """One operand holds small whole numbers, the other such numbers and 2^-12 of others, so that its second plane counts: every product and sum is exact in fp32 and
    so is every logit.  (A pass left out would be off by the second plane's sums, about 2^-12 sqrt(d).)"""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(d + T)
    whole = lambda *s: torch.randint(-7, 8, s, generator=g, device="cuda").float()
    x, W = whole(T, d), whole(V, d)
    low = x if low_in == "x" else W
    low += torch.randint(-15, 16, low.shape, generator=g, device="cuda").float() * 2.0 ** -12
    K = 64
    ids = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(T)]).to(torch.int32)
    print(f"[gpu-case] whole numbers T={T} d={d} V={V} low in {low_in}", flush=True)
    _, _, z = tr.head_distill(x, W, torch.zeros(T, K, device="cuda"), ids, 1.0)
    want = (x.double() @ W.double().T).gather(1, ids.long())
    assert want.abs().max() < 4096 and (want * 4096 == (want * 4096).round()).all()
    assert torch.equal(z.double(), want)


@pytest.mark.parametrize("T,d,V", [(20, 768, 1537), (520, 768, 1537), (520, 512, 33001)])
def test_fp32_errors_as_a_whole(tr, T, d, V):
    """The norm of the errors of z, dx and dW is below 2^-16 of the results': n additions leave about 2^-25 sqrt(n / 2) (2^-19 at n = 3 x 1537, 2^-17.3 at 3 x 33001, whose
    k slices are shorter), the planes 2^-22; a pass left out would leave 2^-13."""
    import torch
    x, W, target, _, _, grad = make(torch.float32, T, d, V, 0, 6)
    target = target.clamp(0, V - 1)
    K = 16
    ids = torch.stack([torch.randperm(V, generator=g_, device="cuda")[:K] for g_ in [torch.Generator(device="cuda").manual_seed(1)] for _ in range(T)]).to(torch.int32)
    print(f"[gpu-case] norms T={T} d={d} V={V}", flush=True)
    _, lse, z = tr.head_distill(x, W, torch.zeros(T, K, device="cuda"), ids, 1.0)
    dx, dW = tr.head_loss_grad(x, W, target, lse, grad)
    Z = x.double() @ W.double().T
    G = torch.exp(Z - torch.logsumexp(Z, 1, keepdim=True))
    G[torch.arange(T, device="cuda"), target.long()] -= 1
    G *= grad.double()[:, None]
    for name, got, want in (("z", z, Z.gather(1, ids.long())), ("dx", dx, G @ W.double()), ("dW", dW, G.T @ x.double())):
        off = ((got.double() - want).norm() / want.norm()).item()
        print(f"HEAD norm {name}: {off:.2e}", flush=True)
        assert off < 2.0 ** -16, name


def test_the_forms_for_few_and_many_fp32_rows_agree(tr):
    """The same rows in a call of 128 (the rows as they are) and of 129 (planes): loss and lse within the sum of both bounds, each within its own."""
    import torch
    x, W, target, _, _, grad = make(torch.float32, 129, 256, 3000, 0, 2)
    print("[gpu-case] fp32 forms", flush=True)
    many, lse_many = tr.head_loss(x, W, target)
    few, lse_few = tr.head_loss(x[:128], W, target[:128].contiguous())
    ex = Exact(x, W, target, None, None, 1.0, grad)
    near("loss of few", few, ex.loss[:128], ex.tol_loss[:128])
    near("loss of many", many, ex.loss, ex.tol_loss)
    near("loss, few and many", few, many[:128].double(), 2 * ex.tol_loss[:128])
    near("lse, few and many", lse_few, lse_many[:128].double(), 2 * ex.tol_lse[:128])


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,d,V,K", [(1, 1, 1, 0), (2, 1, 2, 0), (3, 2, 1, 1), (2, 3, 5, 2), (7, 7, 9, 0), (70, 1, 3, 2), (129, 5, 2, 0), (300, 2, 300, 1)])
def test_smallest_sizes(tr, name, T, d, V, K):
    print(f"[gpu-case] smallest {name} T={T} d={d} V={V} K={K}", flush=True)
    if K:
        distillation_and_gradients(tr, name, T, d, V, K, 1.0)
    else:
        loss_and_gradients(tr, name, T, d, V)


def test_the_last_token_of_a_long_sequence(tr):
    import torch
    states = torch.randn(1, 2000, 4096, device="cuda").bfloat16()
    W, target = torch.randn(500, 4096, device="cuda").bfloat16(), torch.tensor([7], dtype=torch.int32, device="cuda")
    print("[gpu-case] last token", flush=True)
    for a, b in zip(tr.head_loss(states[:, -1], W, target), tr.head_loss(states[0, -1:].clone(), W, target)):
        assert a.isfinite().all() and torch.equal(a, b)
