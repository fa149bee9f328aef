"""Rows that are not contiguous under the head operators: the results are the contiguous rows' bit for bit, and the call's time is of the same order."""
import pytest

from test_gpu_head import make, types

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    import torch
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    tide_route.load_library()
    return tide_route


def spread(a, extra):
    """The same rows, `extra` elements of NaN apart."""
    import torch
    out = torch.full((a.shape[0], a.shape[1] + extra), float("nan"), dtype=a.dtype, device=a.device)
    out[:, :a.shape[1]] = a
    return out[:, :a.shape[1]]


# aligned rows, rows off 16 bytes (hidden sizes that are no whole chunks), few and many of them
@pytest.mark.parametrize("name,T,d,V,extra", [("f32", 20, 64, 400, 8), ("f32", 200, 1024, 700, 4), ("f32", 150, 2052, 300, 12), ("f32", 140, 66, 300, 3), ("f32", 9, 33, 70, 1),
                                              ("f16", 200, 96, 500, 8), ("bf16", 70, 35, 300, 5)])
def test_strided_rows(tr, name, T, d, V, extra):
    import torch
    x, W, target, values, ids, grad = make(types()[name], T, d, V, 5, T + V)
    X, H = spread(x, extra), spread(W, extra)
    print(f"[gpu-case] strided {name} T={T} d={d} V={V} extra={extra}", flush=True)
    want, got = tr.head_loss(x, W, target), tr.head_loss(X, H, target)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    for a, b in zip(tr.head_loss_grad(x, W, target, want[1], grad), tr.head_loss_grad(X, H, target, want[1], grad)):
        assert a.isfinite().all() and torch.equal(a, b)
    want, got = tr.head_distill(x, W, values, ids, 2.0), tr.head_distill(X, H, values, ids, 2.0)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    for a, b in zip(tr.head_distill_grad(x, W, values, ids, 2.0, want[1], grad), tr.head_distill_grad(X, H, values, ids, 2.0, want[1], grad)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("d", [256, 4096])
def test_strided_fp32_rows_take_no_longer(tr, d):
    """The head's rows with a gap between them are dealt out like contiguous ones: within four times their time (a walk through all of them in one
    workgroup is tens of times that)."""
    import torch
    T, V = 256, 32768
    x, W, target, _, _, _ = make(torch.float32, T, d, V, 0, 3)
    H = spread(W, 64)

    def us(weights):
        tr.head_loss(x, weights, target)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        for _ in range(5):
            tr.head_loss(x, weights, target)
        end.record()
        end.synchronize()
        return start.elapsed_time(end) * 200
    print(f"[gpu-case] strided time d={d}", flush=True)
    together, apart = us(W), us(H)
    print(f"HEAD d={d}: contiguous {together:.0f} us, apart {apart:.0f} us", flush=True)
    assert apart < 4 * together
