"""A training iteration's entry points refuse what they cannot take on the host, before any device is touched (no GPU needed)."""
import ctypes

import pytest

import paper_2008_12260_amd as px

FAKE = ctypes.c_void_p(0x10000)          # never dereferenced: validation, or the device check, fails first
ODD = ctypes.c_void_p(0x10008)
NULL = ctypes.c_void_p(0)


def refused(call, dims, args, changes, code):
    """Each (position, value) alone makes the call fail with `code`; position -1 replaces the dims."""
    for at, value in changes:
        bad = list(args)
        if at < 0:
            assert call(None if value is None else ctypes.byref(value), *bad) == code, value
        else:
            bad[at] = value
            assert call(ctypes.byref(dims), *bad) == code, (at, value)


def loss_dims(**changes):
    d = px.LossDims(64, 1000, 128, px.PX_TYPE_BF16, 0, 0, 0, 0, 0)
    for k, v in changes.items():
        setattr(d, k, v)
    return d


BAD_LOSS_DIMS = [dict(N=-1), dict(N=(1 << 20) + 1), dict(V=0), dict(V=(1 << 20) + 1), dict(D=0), dict(D=(1 << 16) + 1), dict(type=3), dict(type=-1),
                 dict(flags=4), dict(hidden_stride=127), dict(weight_stride=-1), dict(weight_stride=1 << 20), dict(hidden_grad_stride=5),
                 dict(weight_grad_stride=1)]


def test_loss_workspace():
    L, n = px.lib(), ctypes.c_size_t()

    def size(d, grad):
        assert L.pollux_loss_workspace_size(ctypes.byref(d), grad, ctypes.byref(n)) == px.PX_OK
        return n.value

    assert 0 < size(loss_dims(), 0) < size(loss_dims(), 1)
    assert size(loss_dims(N=0), 1) > 0
    # logits of 8192 tokens over 131072 entries in bfloat16 would be 2 GiB
    assert size(loss_dims(N=8192, V=131072, D=4096), 0) < 1 << 28
    assert size(loss_dims(N=8192, V=131072, D=4096), 1) < 2 << 30
    for grad in (2, -1):
        assert L.pollux_loss_workspace_size(ctypes.byref(loss_dims()), grad, ctypes.byref(n)) == px.PX_E_INVALID_ARG
    assert L.pollux_loss_workspace_size(ctypes.byref(loss_dims()), 0, None) == px.PX_E_INVALID_ARG
    for change in BAD_LOSS_DIMS:
        assert L.pollux_loss_workspace_size(ctypes.byref(loss_dims(**change)), 0, ctypes.byref(n)) == px.PX_E_INVALID_ARG, change


def test_loss_refusals():
    L, d = px.lib(), loss_dims()
    bad_dims = [(-1, None)] + [(-1, loss_dims(**c)) for c in BAD_LOSS_DIMS]
    # hidden, weight, targets, workspace, bytes, loss, lse, stream
    forward = [FAKE, FAKE, FAKE, FAKE, 1 << 40, FAKE, FAKE, NULL]
    refused(L.pollux_token_loss, d, forward, bad_dims + [(0, NULL), (1, NULL), (2, NULL), (5, NULL), (6, NULL), (0, ODD), (1, ODD)], px.PX_E_INVALID_ARG)
    refused(L.pollux_token_loss, d, forward, [(3, NULL), (3, ODD), (4, 16)], px.PX_E_WORKSPACE)
    # hidden, weight, targets, lse, row_weight, workspace, bytes, hidden_grad, weight_grad, stream
    backward = [FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, FAKE, FAKE, NULL]
    refused(L.pollux_token_loss_grad, d, backward, bad_dims + [(0, NULL), (1, NULL), (2, NULL), (3, NULL), (0, ODD), (1, ODD), (7, ODD), (8, ODD)],
            px.PX_E_INVALID_ARG)
    refused(L.pollux_token_loss_grad, d, backward, [(5, NULL), (5, ODD), (6, 16)], px.PX_E_WORKSPACE)


def test_tensors_that_are_not_on_a_gpu_are_refused():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("a GPU is there")
    with pytest.raises((RuntimeError, ValueError, AssertionError)):
        px.token_loss(torch.zeros((2, 8)), torch.zeros((4, 8)), torch.zeros(2, dtype=torch.int64))
