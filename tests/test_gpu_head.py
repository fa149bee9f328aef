"""The head operators (loss, distillation, their gradients) against the formulas in 64 bits on the device.

Tolerances are bounds, derived term by term from the arithmetic (u = half a step of the storage type, e = 2^-24):
  z       products of 16-bit values are exact, d additions in fp32: d e sum|x W|.  fp32 operands are pairs of fp16 values, each off by at most
          2^-23 of the value (2 of them), the dropped product of the small halves is 2^-22 at most: 2^-21 sum|x W| more, and
          2^-38 of the largest magnitudes' product per term where a small half is below fp16's range
  lse     the error of z / tau, and exp2 / log2 and their arguments' roundings: 2^-20 (1 + |lse|)
  G       u |G| for its rounding, g tau p (twice the above) for the exponential, e g tau q; fp16: 2^-38 max|g tau| below its range
  dx, dW  the error of G through the product, the additions in fp32, u of the result for its rounding
The inputs leave rows without a target, hold NaN in such rows, and repeat and misplace the teacher's tokens."""
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
NAMES = ("f32", "f16", "bf16")


@pytest.fixture(scope="module")
def tr():
    import torch
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    tide_route.load_library()
    return tide_route


def types():
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def half_step(dtype):
    import torch
    return torch.finfo(dtype).eps / 2


def make(dtype, T, d, V, K, seed, spread=1.5):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    W = (torch.randn(V, d, generator=g, device="cuda") * (spread / d ** 0.5)).to(dtype)
    x = torch.randn(T, d, generator=g, device="cuda")
    target = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    x = (x + 3.0 * W[target.long()].float()).to(dtype)
    if T > 2:
        target[1], target[T // 2], target[T - 1] = -1, V, -2147483648      # three kinds of no target
    grad = 0.5 + torch.rand(T, generator=g, device="cuda")
    if T > 5:
        grad[4] = 0.0
    if not K:
        return x, W, target, None, None, grad
    ids = torch.randint(0, V, (T, K), generator=g, device="cuda", dtype=torch.int32)
    ids[:, 0] = target.clamp(0, V - 1)
    values = 4.0 * torch.randn(T, K, generator=g, device="cuda")
    if T > 3:
        ids[1] = -1                                    # no entry at all
        values[2] = -float("inf")                      # entries, but none that counts
        ids[3, K // 2:] = V + 5
        if K > 2:
            ids[0, 2] = ids[0, 0]                      # a token given twice
            values[0, 1] = -float("inf")
    return x, W, target, values, ids, grad


class Exact:
    """The formulas in 64 bits, and the bounds on what 32-bit arithmetic may be off by."""

    def __init__(self, x, W, target, values, ids, tau, grad, lse=None):
        import torch
        T, V, d, dtype = x.shape[0], W.shape[0], x.shape[1], x.dtype
        x, W = x.double(), W.double()
        self.z = x @ W.T
        size = x.abs() @ W.abs().T
        self.tol_z = d * E * size
        if dtype == torch.float32:
            finite = x[x.isfinite()]
            self.tol_z += 2.0 ** -21 * size + d * 2.0 ** -38 * (finite.abs().max() if finite.numel() else 0.0) * W.abs().max()
        y = self.z / tau
        self.lse = torch.logsumexp(y, 1)
        tol_y = self.tol_z.amax(1) / tau
        self.tol_lse = tol_y + 2.0 ** -20 * (1 + self.lse.abs())
        teacher = torch.zeros_like(self.z)
        if values is None:
            there = (target >= 0) & (target < V)
            t = there.nonzero()[:, 0]
            teacher[t, target[t].long()] = 1.0
            self.live = there
            zy = torch.zeros_like(self.lse)
            zy[t] = self.z[t, target[t].long()]
            self.loss = torch.where(there, self.lse - zy, 0.0)
            self.tol_loss = self.tol_lse + tol_y + 2 * E * zy.abs()
        else:
            there = (ids >= 0) & (ids < V) & (values != -float("inf"))
            v = values.double().masked_fill(~there, -float("inf")) / tau
            q = torch.nan_to_num(torch.softmax(v, 1), nan=0.0)
            inside = (ids >= 0) & (ids < V)
            at = torch.where(inside, ids, 0).long()
            self.z_top = torch.where(inside, self.z.gather(1, at), 0.0)
            self.tol_top = torch.where(inside, self.tol_z.gather(1, at), 0.0)
            teacher.scatter_add_(1, at, q)
            self.live = there.any(1)
            log_q = torch.where(q > 0, torch.log(torch.where(q > 0, q, 1.0)), 0.0)
            terms = q * (log_q - self.z_top / tau + self.lse[:, None])
            self.loss = torch.where(self.live, tau * tau * terms.sum(1), 0.0)
            size = (q * (log_q.abs() + self.z_top.abs() / tau + self.lse.abs()[:, None])).sum(1)
            spread = torch.where(there, v.abs(), 0.0).amax(1)
            self.tol_loss = tau * tau * (self.tol_lse + tol_y + (ids.shape[1] + 16 + 4 * spread) * E * size)
        self.teacher, self.tau, self.dtype, self.x, self.W, self.grad = teacher, tau, dtype, x, W, grad.double()
        self.tol_p = 2 * (tol_y + self.tol_lse)

    def gradients(self, kept):
        """dx, dW and their bounds; `kept`: the loss's rows that have a gradient."""
        import torch
        g = torch.where(kept, self.grad * self.tau, 0.0)[:, None]
        x = torch.where(kept[:, None], self.x, 0.0)
        p = torch.where(kept[:, None], torch.exp(self.z / self.tau - self.lse[:, None]), 0.0)
        G = g * (p - torch.where(kept[:, None], self.teacher, 0.0))
        u = half_step(self.dtype)
        gu = {torch.float32: 2.0 ** -22, torch.float16: u, torch.bfloat16: u}[self.dtype]
        tol_G = gu * G.abs() + g.abs() * (p * self.tol_p.nan_to_num(0.0)[:, None] + 16 * E * (p + self.teacher))
        if self.dtype != torch.bfloat16:
            tol_G = tol_G + 2.0 ** -38 * g.abs().max()
        plane = 2.0 ** -22 if self.dtype == torch.float32 else 0.0
        out = []
        for A, tol_A, B in ((G, tol_G, self.W), (G.T, tol_G.T, x)):
            n = A.shape[1]
            exact, size = A @ B, A.abs() @ B.abs()
            floor = n * 2.0 ** -38 * A.abs().max() * B.abs().max() if self.dtype == torch.float32 else 0.0
            out += [exact, tol_A @ B.abs() + (n * E + plane) * size + floor + u * 1.01 * exact.abs() + (2.0 ** -25 if self.dtype == torch.float16 else 1e-38)]
        return out


def near(name, got, want, tol):
    import torch
    got = got.double()
    assert torch.isfinite(got).all(), f"{name}: not finite"
    off = (got - want).abs()
    worst = ((off - tol) > 0).sum().item()
    print(f"HEAD {name}: largest difference {off.max().item() if off.numel() else 0:.3e}, largest share of its bound {(off / tol.clamp(min=1e-300)).max().item() if off.numel() else 0:.3f}", flush=True)
    assert worst == 0, f"{name}: {worst} values beyond their bounds"


# (T, d, V): one row and few, every tile height and its edges, hidden sizes from 8 bytes to no multiple of anything, one token, odd vocabularies
SIZES = [(1, 64, 1000), (1, 8, 1), (17, 72, 257), (31, 1600, 255), (33, 128, 513), (64, 40, 7), (65, 256, 1030), (128, 96, 256), (129, 100, 511), (200, 64, 2),
         (257, 512, 777), (300, 33, 4099), (520, 768, 1537), (640, 200, 300)]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("T,d,V", SIZES)
def test_loss_and_gradients(tr, name, T, d, V):
    import torch
    dtype = types()[name]
    x, W, target, _, _, grad = make(dtype, T, d, V, 0, 7 * T + d + V)
    if T > 5:
        x[1], x[4, 0] = float("nan"), float("inf")     # rows that have no gradient
    print(f"[gpu-case] loss {name} T={T} d={d} V={V}", flush=True)
    loss, lse = tr.head_loss(x, W, target)
    torch.cuda.synchronize()
    clean = x.clone()
    if T > 5:
        clean[1], clean[4] = 0.0, 0.0
    ex = Exact(clean, W, target, None, None, 1.0, grad)
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    if T > 5:
        rows[1] = rows[4] = False
        assert loss[1] == 0 and lse[1].isnan()
    near("lse", lse[rows], ex.lse[rows], ex.tol_lse[rows])
    near("loss", loss[rows], ex.loss[rows], ex.tol_loss[rows])
    print("[gpu-case] gradients", flush=True)
    dx, dW = tr.head_loss_grad(x, W, target, lse, grad)
    torch.cuda.synchronize()
    kept = ex.live & (grad != 0)
    want_dx, tol_dx, want_dw, tol_dw = ex.gradients(kept)
    assert dx.dtype == dW.dtype == dtype and (dx[~kept] == 0).all()
    near("dx", dx, want_dx, tol_dx)
    near("dW", dW, want_dw, tol_dw)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("T,d,V,K,tau", [(1, 64, 1000, 1, 1.0), (5, 72, 300, 3, 2.0), (40, 128, 257, 8, 0.5), (70, 100, 1000, 32, 4.0), (130, 256, 90, 128, 2.0), (300, 512, 1500, 33, 1.0),
                                         (520, 64, 513, 200, 3.0)])
def test_distillation_and_gradients(tr, name, T, d, V, K, tau):
    import torch
    dtype = types()[name]
    x, W, _, values, ids, grad = make(dtype, T, d, V, K, 11 * T + d + V + K)
    print(f"[gpu-case] distill {name} T={T} d={d} V={V} K={K} tau={tau}", flush=True)
    loss, lse, z = tr.head_distill(x, W, values, ids, tau)
    torch.cuda.synchronize()
    ex = Exact(x, W, None, values, ids, tau, grad)
    near("lse", lse, ex.lse, ex.tol_lse)
    near("z", z, ex.z_top, ex.tol_top + 1e-300)
    near("loss", loss, ex.loss, ex.tol_loss)
    print("[gpu-case] gradients", flush=True)
    dx, dW = tr.head_distill_grad(x, W, values, ids, tau, lse, grad)
    torch.cuda.synchronize()
    kept = ex.live & (grad != 0)
    want_dx, tol_dx, want_dw, tol_dw = ex.gradients(kept)
    assert (dx[~kept] == 0).all()
    near("dx", dx, want_dx, tol_dx)
    near("dW", dW, want_dw, tol_dw)


@pytest.mark.parametrize("name", NAMES)
def test_several_pieces_of_the_vocabulary(tr, name):
    """So many rows that the gradient goes through the vocabulary in pieces, the last one ragged."""
    import torch
    T, d, V = {"f32": (6000, 64, 20011), "f16": (8200, 72, 20011), "bf16": (8200, 72, 40003)}[name]
    x, W, target, _, _, grad = make(types()[name], T, d, V, 0, 5)
    print(f"[gpu-case] pieces {name} T={T} V={V}", flush=True)
    loss, lse = tr.head_loss(x, W, target)
    dx, dW = tr.head_loss_grad(x, W, target, lse, grad)
    torch.cuda.synchronize()
    ex = Exact(x, W, target, None, None, 1.0, grad)
    near("loss", loss, ex.loss, ex.tol_loss)
    want_dx, tol_dx, want_dw, tol_dw = ex.gradients(ex.live & (grad != 0))
    near("dx", dx, want_dx, tol_dx)
    near("dW", dW, want_dw, tol_dw)


def test_strided_rows_and_one_product(tr):
    import torch
    T, d, V = 70, 64, 400
    x, W, target, _, _, grad = make(torch.bfloat16, T, d, V, 0, 3)
    X = torch.full((T, d + 24), float("nan"), dtype=x.dtype, device="cuda")
    H = torch.full((V, d + 8), float("nan"), dtype=x.dtype, device="cuda")
    X[:, :d], H[:, :d] = x, W
    print("[gpu-case] strided rows", flush=True)
    want = tr.head_loss(x, W, target)
    got = tr.head_loss(X[:, :d], H[:, :d], target)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    both = tr.head_loss_grad(x, W, target, want[1], grad)
    dx, none = tr.head_loss_grad(X[:, :d], H[:, :d], target, want[1], grad, want_dw=False)
    assert none is None and torch.equal(dx, both[0])
    none, dW = tr.head_loss_grad(X[:, :d], H[:, :d], target, want[1], grad, want_dx=False)
    assert none is None and torch.equal(dW, both[1])


def test_no_rows_and_no_live_rows(tr):
    import torch
    W = torch.randn(300, 64, device="cuda").bfloat16()
    empty = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    f = lambda n: torch.ones(n, device="cuda")
    print("[gpu-case] no rows", flush=True)
    loss, lse = tr.head_loss(empty, W, torch.empty(0, dtype=torch.int32, device="cuda"))
    assert loss.numel() == lse.numel() == 0
    dx, dW = tr.head_loss_grad(empty, W, torch.empty(0, dtype=torch.int32, device="cuda"), f(0), f(0))
    assert dx.shape == (0, 64) and (dW == 0).all()
    x = torch.full((40, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    print("[gpu-case] no live rows", flush=True)
    dx, dW = tr.head_loss_grad(x, W, torch.full((40,), -1, dtype=torch.int32, device="cuda"), f(40), f(40))
    assert (dx == 0).all() and (dW == 0).all()


def test_repeated_calls_give_the_same_bits_on_any_stream_and_workspace(tr):
    import torch
    x, W, target, values, ids, grad = make(torch.float16, 300, 256, 3001, 9, 12)
    loss, lse, z = tr.head_distill(x, W, values, ids, 2.0)
    first = (loss, lse, z, *tr.head_distill_grad(x, W, values, ids, 2.0, lse, grad))
    torch.cuda.synchronize()
    ws = torch.full((tr.head_workspace_bytes(tr.F16, 300, 256, 3001, 9, gradient=True),), 0xff, dtype=torch.uint8, device="cuda")     # (0xffff: a NaN)
    side = torch.cuda.Stream()
    print("[gpu-case] another stream, a workspace of NaN", flush=True)
    with torch.cuda.stream(side):
        a = tr.head_distill(x, W, values, ids, 2.0)
        b = tr.head_distill_grad(x, W, values, ids, 2.0, lse, grad, workspace=ws)
    side.synchronize()
    for p, q in zip(first, (*a, *b)):
        assert torch.equal(p, q)


def test_captured_in_a_graph(tr):
    """A step replayed on new inputs gives the eager step's bits, with eager work between the replays."""
    import torch
    make_one = lambda seed: make(torch.bfloat16, 100, 128, 2000, 0, seed)
    x, W, target, _, _, grad = make_one(1)

    def step():
        loss, lse = tr.head_loss(x, W, target)
        return (loss, lse, *tr.head_loss_grad(x, W, target, lse, grad))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    print("[gpu-case] graph", flush=True)
    with torch.cuda.graph(graph):
        out = step()
    for seed in (2, 3, 4):
        for to, new in zip((x, W, target, grad), (lambda m: (m[0], m[1], m[2], m[5]))(make_one(seed))):
            to.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b)


def test_gradient_against_differences(tr):
    """dx and dW of the summed loss against central differences of the fp32 forward call."""
    import torch
    T, d, V = 24, 32, 90
    x, W, target, _, _, grad = make(torch.float32, T, d, V, 0, 21)
    loss, lse = tr.head_loss(x, W, target)
    dx, dW = tr.head_loss_grad(x, W, target, lse, grad)
    total = lambda a, b: (tr.head_loss(a, b, target)[0].double() * grad.double()).sum().item()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    print("[gpu-case] differences", flush=True)
    for _ in range(4):
        u, w = torch.randn(T, d, generator=g, device="cuda"), torch.randn(V, d, generator=g, device="cuda")
        h = 2.0 ** -7
        got = (total(x + h * u, W + h * w) - total(x - h * u, W - h * w)) / (2 * h)
        want = (dx.double() * u).sum().item() + (dW.double() * w).sum().item()
        # third-order term of the loss along a direction of this size, times h^2, and the losses' own errors over h
        assert abs(got - want) < h * h * 60 * T + T * 4.0 * 2.0 ** -17 / h * 0.01 + 1e-3 * abs(want), (got, want)


PROJECT = [("bf16", 3, 1, 4096), ("f16", 4, 37, 512), ("f32", 2, 700, 1600), ("bf16", 3, 1100, 72), ("f32", 2, 5, 16384), ("bf16", 1, 9, 16384)]


@pytest.mark.parametrize("name,C,T,d", PROJECT)
@pytest.mark.parametrize("with_final", [True, False])
def test_projection_gradient(tr, name, C, T, d, with_final):
    import torch
    dtype = types()[name]
    g = torch.Generator(device="cuda")
    g.manual_seed(T + d)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    hidden, final, dy = (3 * rand(C, T, d)).to(dtype), rand(T, d).to(dtype), rand(T, d).to(dtype)
    ids = [4 * c + 3 for c in range(C)]
    exits = (4 * torch.randint(0, C + 1, (T,), generator=g, device="cuda") + 3).to(torch.int32)
    gain, eps = 1 + 0.1 * rand(d), 1e-5
    print(f"[gpu-case] project_grad {name} C={C} T={T} d={d} final={with_final}", flush=True)
    grad, dgain = tr.exit_project_grad(hidden, final if with_final else None, exits, ids, gain, eps, dy)
    torch.cuda.synchronize()
    at = (exits.long() - 3) // 4
    src = torch.cat((hidden, final[None]))[at, torch.arange(T, device="cuda")].double()
    there = torch.ones_like(at, dtype=torch.bool) if with_final else at < C
    src = torch.where(there[:, None], src, 1.0).requires_grad_()
    gd = gain.double().requires_grad_()
    y = src * torch.rsqrt((src * src).mean(1, keepdim=True) + eps) * gd
    y.backward(torch.where(there[:, None], dy.double(), 0.0))
    # d additions in each of the two sums, a dozen roundings around them; the result's own
    r = torch.rsqrt((src * src).mean(1, keepdim=True) + eps).detach()
    n, u = src.detach() * r, torch.where(there[:, None], dy.double(), 0.0) * gain.double()
    size = r * (u.abs() + n.abs() * (u * n).abs().mean(1, keepdim=True))
    near("grad", grad, src.grad, (d + 12) * E * size + half_step(dtype) * 1.01 * src.grad.abs() + 2.0 ** -25)
    near("gain", dgain, gd.grad, (T + d + 12) * E * (dy.double() * n).abs().sum(0) + 1e-30)
    if not with_final:
        assert (grad[~there] == 0).all()
    again, none = tr.exit_project_grad(hidden, final if with_final else None, exits, ids, gain, eps, dy, want_gain=False)
    assert none is None and torch.equal(again, grad)
