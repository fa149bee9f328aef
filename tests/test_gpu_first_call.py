"""A first call, which allocates and clears the library's workspace, on a stream of its own while the null stream is busy: the clearing is done when the call's kernels run."""
import pytest

from paper_2603_21365_amd import synth
from parity import routers_to_device, to_device

pytestmark = pytest.mark.gpu


@pytest.fixture
def tr():
    import torch
    assert torch.cuda.is_available()
    from paper_2603_21365_amd import tide_route
    yield tide_route
    tide_route.release()


def busy():
    """Some 50 ms of work on the null stream, enqueued."""
    import torch
    a = torch.ones(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    for _ in range(8):
        a @ a


def test_router_calls(tr):
    import torch
    w = synth.Workload("first_call", 109, "bf16", 256, 8, 4, 3100, None)
    h, rt = to_device(w.hidden(), "bf16"), w.routers()
    g, W1, b1, w2 = routers_to_device(rt)
    packed = tr.router_pack(tr.BF16, g, W1)
    call = lambda: tr.select_exit_packed(h, packed, w.eps, b1, w2, rt.b2, rt.theta, w.layer_ids, 0, w.n_layers, d=256)
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    tr.release()
    print("[gpu-case] first router call behind a busy null stream", flush=True)
    busy()
    with torch.cuda.stream(side):
        got = [call() for _ in range(3)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got.append(call())
    side.synchronize()
    for out in got:
        assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_batch_calls(tr):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    C, T, ids = 4, 50000, [3, 7, 11, 15]
    exits = (4 * torch.randint(0, C + 1, (T,), generator=g, device="cuda") + 3).to(torch.int32)
    mask = (torch.randint(0, 1 << C, (T,), generator=g, device="cuda") | 2).to(torch.int32)
    calls = (lambda: tr.batch_exit(mask, C, ids, 0, 16), lambda: tr.batch_compact(exits, 7))
    for call in calls:
        want = call()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        tr.release()
        print("[gpu-case] first batch call behind a busy null stream", flush=True)
        busy()
        with torch.cuda.stream(side):
            got = [call() for _ in range(3)]
        torch.cuda.synchronize()
        for out in got:
            assert all(torch.equal(x, y) for x, y in zip(out, want) if isinstance(x, torch.Tensor))
