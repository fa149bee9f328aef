"""What the head operators and the projection's gradient refuse, before anything is enqueued (no GPU needed), and the size of their workspace."""
import ctypes

import pytest

from paper_2603_21365_amd import tide_route as tr

FAKE = 0x100000     # never dereferenced: every call below fails its checks first
OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 0, -1, -2, -3, -4


def loss(x=FAKE, dtype=2, T=4, d=64, V=100, xs=64, W=FAKE, ws=64, target=FAKE, loss=FAKE, lse=FAKE, space=FAKE, nbytes=0):
    return tr.load_library().tide_head_loss(x, dtype, T, d, V, xs, W, ws, target, loss, lse, space, nbytes, None)


def loss_grad(x=FAKE, dtype=2, T=4, d=64, V=100, xs=64, W=FAKE, ws=64, target=FAKE, lse=FAKE, g=FAKE, dx=FAKE, dxs=64, dW=FAKE, dws=64, space=FAKE, nbytes=0):
    return tr.load_library().tide_head_loss_grad(x, dtype, T, d, V, xs, W, ws, target, lse, g, dx, dxs, dW, dws, space, nbytes, None)


def distill(x=FAKE, dtype=2, T=4, d=64, V=100, W=FAKE, values=FAKE, ids=FAKE, K=3, tau=1.0, loss=FAKE, lse=FAKE, z=FAKE, space=FAKE, nbytes=0):
    return tr.load_library().tide_head_distill(x, dtype, T, d, V, d, W, d, values, ids, K, tau, loss, lse, z, space, nbytes, None)


def distill_grad(K=3, tau=1.0, lse=FAKE, g=FAKE, values=FAKE):
    return tr.load_library().tide_head_distill_grad(FAKE, 2, 4, 64, 100, 64, FAKE, 64, values, FAKE, K, tau, lse, g, FAKE, 64, FAKE, 64, FAKE, 0, None)


@pytest.mark.parametrize("call", [loss, loss_grad])
@pytest.mark.parametrize("bad,status,word", [
    (dict(dtype=3), INVALID, "dtype"), (dict(T=-1), INVALID, "negative"), (dict(T=1 << 23), UNSUPPORTED, "exceeds"), (dict(d=0), INVALID, "positive"),
    (dict(d=16392, xs=16392, ws=16392), UNSUPPORTED, "16384"), (dict(V=0), INVALID, "V = 0"), (dict(V=1 << 24), UNSUPPORTED, "V ="), (dict(T=1 << 22, V=1 << 20), UNSUPPORTED, "too many"), (dict(x=None), INVALID, "NULL"),
    (dict(W=None), INVALID, "NULL"), (dict(target=None), INVALID, "NULL"), (dict(lse=None), INVALID, "lse"), (dict(xs=63), INVALID, "strides"), (dict(ws=63), INVALID, "strides"),
    (dict(xs=1 << 23), UNSUPPORTED, "strides"), (dict(x=FAKE + 8), ALIGNMENT, "x:"), (dict(ws=68), ALIGNMENT, "W:"), (dict(d=63, W=FAKE + 1), ALIGNMENT, "W:"),
    (dict(target=FAKE + 2), ALIGNMENT, "4-byte")])
def test_loss_refusals(call, bad, status, word):
    assert call(**bad) == status and word in tr.last_error()


@pytest.mark.parametrize("bad,status,word", [(dict(g=None), INVALID, "grad_loss"), (dict(dxs=63), INVALID, "dx"), (dict(dws=60), INVALID, "dW"),
                                             (dict(dx=FAKE + 2), ALIGNMENT, "dx"), (dict(dws=66), ALIGNMENT, "dW")])
def test_gradient_refusals(bad, status, word):
    assert loss_grad(**bad) == status and word in tr.last_error()


@pytest.mark.parametrize("bad,status,word", [(dict(K=0), INVALID, "K"), (dict(K=1025), UNSUPPORTED, "K"), (dict(tau=0.0), INVALID, "tau"), (dict(tau=-1.0), INVALID, "tau"),
                                             (dict(tau=float("nan")), INVALID, "tau"), (dict(tau=float("inf")), INVALID, "tau"), (dict(values=None), INVALID, "top_values"),
                                             (dict(z=None), INVALID, "z")])
def test_distillation_refusals(bad, status, word):
    assert distill(**bad) == status and word in tr.last_error()
    if set(bad) <= {"K", "tau", "values"}:
        assert distill_grad(**bad) == status and word in tr.last_error()


def test_no_rows_is_no_work():
    assert loss(T=0, x=None, target=None, loss=None, lse=None, space=None) == OK
    assert loss_grad(dx=None, dW=None) == OK           # neither product is asked for


def test_workspace_sizes():
    size = tr.head_workspace_bytes
    assert size(tr.BF16, 1, 4096, 128000) % 256 == 0 and 0 < size(tr.BF16, 1, 4096, 128000) < 1 << 20
    # the gradient's holds a piece of the vocabulary, not T x V logits
    assert size(tr.BF16, 8192, 4096, 128000, gradient=True) < 8192 * 128000 * 2 // 3
    assert size(tr.F16, 100, 100, 1000) > size(tr.F16, 100, 104, 1000)             # rows that are no whole chunks are copied
    assert size(tr.F32, 17, 768, 32003) < 1 << 20 < 32003 * 768 * 4 < size(tr.F32, 129, 768, 32003)      # few fp32 rows: no planes
    assert size(7, 4, 64, 100) == 0 and "dtype" in tr.last_error()
    assert size(tr.F32, 4, 64, 100, 2000) == 0 and "K" in tr.last_error()
    for T in (0, 1, 31, 33, 64, 65, 129, 193, 257, 4000):      # more of anything never needs less
        assert size(tr.F16, T, 512, 5000, gradient=True) <= size(tr.F16, T + 1, 512, 5000, gradient=True)


def project(dtype=2, C=2, T=4, d=64, hidden=FAKE, exits=FAKE, g=FAKE, grad=FAKE, gain_out=FAKE, gs=64, rs=64, final=None, frs=64, norm=None, space=None, nbytes=0, ids=(3, 7)):
    host = (ctypes.c_int32 * len(ids))(*ids)
    return tr.load_library().tide_exit_project_grad(hidden, dtype, C, T, d, T * d, d, final, frs, exits, host, norm, 1e-6, g, gs, grad, rs, gain_out, space, nbytes, None)


@pytest.mark.parametrize("bad,status,word", [
    (dict(dtype=9), INVALID, "dtype"), (dict(C=33, ids=tuple(range(33))), UNSUPPORTED, "32"), (dict(d=33), UNSUPPORTED, "16 bytes"), (dict(hidden=None), INVALID, "NULL"),
    (dict(exits=None), INVALID, "NULL"), (dict(g=None), INVALID, "NULL"), (dict(grad=None), INVALID, "NULL"), (dict(gs=60), INVALID, "strides"), (dict(rs=60), INVALID, "strides"),
    (dict(final=FAKE, frs=60), INVALID, "strides"), (dict(gs=66), ALIGNMENT, "multiples"), (dict(grad=FAKE + 8), ALIGNMENT, "multiples"), (dict(norm=FAKE + 4), ALIGNMENT, "multiples"),
    (dict(gain_out=FAKE + 2), ALIGNMENT, "grad_gain"), (dict(ids=(7, 7)), INVALID, "ascending")])
def test_projection_gradient_refusals(bad, status, word):
    assert project(**bad) == status and word in tr.last_error()


def test_projection_gradient_workspace():
    size = tr.load_library().tide_exit_project_grad_bytes
    assert size(1, 4096) == 16384 and size(8192, 4096) == 1024 * 4096 * 4 and size(-1, 64) == 0 and size(4, 20000) == 0
