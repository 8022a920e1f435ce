"""A training iteration's operators on torch device tensors (C ABI in include/pollux.h, "A training iteration of a
language-model job"): what a job's agent runs to obtain the gradients whose noise scale, and the iterations whose times,
the scheduler is given.

Arguments are checked and marshalled here; every step runs in the library's kernels.  Results and scratch memory are allocated
by torch on the stream that the call is enqueued on (`stream`, else the current one); nothing synchronises, so the calls
can be recorded into a graph.  A caller who hands over results or scratch memory from another stream keeps them in order, as with any
torch operation.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

import paper_2008_12260_amd as _px


def _types():
    import torch
    return {torch.float32: _px.PX_TYPE_F32, torch.bfloat16: _px.PX_TYPE_BF16, torch.float16: _px.PX_TYPE_F16}


def _type(t, name):
    code = _types().get(t.dtype)
    if code is None:
        raise TypeError(f"{name} is {t.dtype}: float32, bfloat16 or float16 is wanted")
    return code


def _on_device(**tensors):
    """All given tensors on the current GPU: the library launches there, and reads what it is given there."""
    import torch
    here = torch.cuda.current_device()
    for name, t in tensors.items():
        if t is not None and (not t.is_cuda or t.device.index != here):
            raise ValueError(f"{name} is on {t.device}: it has to be on the current GPU, cuda:{here}")


def _rows(t, name):
    """(the tensor, its stride in elements): a matrix whose rows are contiguous and begin at a multiple of 16 bytes, as it is or copied."""
    if t.dim() != 2:
        raise ValueError(f"{name} has {t.dim()} dimensions: 2 are wanted")
    if t.shape[1] > 1 and t.stride(1) != 1 or t.shape[0] > 1 and (t.stride(0) < t.shape[1] or t.stride(0) >= 1 << 20) or t.data_ptr() % 16:
        t = t.clone(memory_format=_contiguous())
    return t, t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _contiguous():
    import torch
    return torch.contiguous_format


def _result(t, name, shape, dtype):
    """(a caller's result, its stride): written in place, so it has to be as the library takes it."""
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype} {tuple(t.shape)}: {dtype} {tuple(shape)} is wanted")
    if t.shape[1] > 1 and t.stride(1) != 1 or t.shape[0] > 1 and t.stride(0) < t.shape[1] or t.data_ptr() % 16:
        raise ValueError(f"{name} needs contiguous rows and a base aligned to 16 bytes")
    return t, t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _tokens(t, name, count):
    """(the tensor, its flag): int64 or int32, one for each row."""
    import torch
    if t.dtype not in (torch.int64, torch.int32):
        raise TypeError(f"{name} is {t.dtype}: int64 or int32 is wanted")
    if t.numel() != count:
        raise ValueError(f"{name} has {t.numel()} elements for {count} rows")
    return t.contiguous(), _px.PX_FLAG_TOKENS_I64 if t.dtype == torch.int64 else 0


def _on(stream):
    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _scratch(bytes_, device):
    import torch
    ws = torch.empty(bytes_, dtype=torch.uint8, device=device)
    if os.environ.get("POLLUX_POISON_WORKSPACE"):
        # for tests: nothing in the library may depend on what a fresh workspace holds (0xFF bytes read as NaN / -1)
        ws.fill_(0xFF)
    return ws


def _check(rc, where):
    if rc != _px.PX_OK:
        raise _px.PolluxError(rc, where)


def _loss_call(hidden, weight, targets):
    _on_device(hidden=hidden, weight=weight, targets=targets)
    if hidden.dtype != weight.dtype:
        raise TypeError(f"hidden is {hidden.dtype} and weight {weight.dtype}: one type is wanted")
    type_ = _type(hidden, "hidden")
    hidden, hidden_stride = _rows(hidden, "hidden")
    weight, weight_stride = _rows(weight, "weight")
    if hidden.shape[1] != weight.shape[1]:
        raise ValueError(f"rows of hidden have {hidden.shape[1]} elements, of weight {weight.shape[1]}")
    targets, flag = _tokens(targets, "targets", hidden.shape[0])
    dims = _px.LossDims(hidden.shape[0], weight.shape[0], hidden.shape[1], type_, flag, hidden_stride, weight_stride, 0, 0)
    return dims, hidden, weight, targets


def _loss_scratch(dims, grad, workspace, device):
    need = ctypes.c_size_t(0)
    _check(_px.lib().pollux_loss_workspace_size(ctypes.byref(dims), grad, ctypes.byref(need)), "pollux_loss_workspace_size")
    return _scratch(need.value, device) if workspace is None else workspace


def token_loss(hidden, weight, targets, workspace=None, stream=None):
    """Cross entropy of each row of `hidden` [N, D] over the vocabulary that `weight` [V, D] projects to: (loss [N], lse [N]), fp32.

    targets [N], int64 or int32; -1 is none (loss 0), anything else outside the vocabulary too, reported by
    pollux_last_status(workspace) where the caller gives the workspace."""
    import torch
    with _on(stream):
        dims, hidden, weight, targets = _loss_call(hidden, weight, targets)
        workspace = _loss_scratch(dims, 0, workspace, hidden.device)
        loss = torch.empty(dims.N, dtype=torch.float32, device=hidden.device)
        lse = torch.empty(dims.N, dtype=torch.float32, device=hidden.device)
        _check(_px.lib().pollux_token_loss(ctypes.byref(dims), hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), workspace.data_ptr(),
                                           workspace.numel() * workspace.element_size(), loss.data_ptr(), lse.data_ptr(),
                                           _px._stream_handle(stream)), "pollux_token_loss")
    return loss, lse


def token_loss_grad(hidden, weight, targets, lse, row_weight=None, hidden_grad=None, weight_grad=None, accumulate=False, need=(True, True),
                    workspace=None, stream=None):
    """Gradients of sum_n row_weight[n] * loss[n] with respect to `hidden` and `weight`, in their type: (hidden_grad [N, D],
    weight_grad [V, D]), None for one that is not needed.

    lse: of token_loss on the same arguments; row_weight [N] fp32, or None for ones.  accumulate: weight_grad is given and
    added to."""
    import torch
    with _on(stream):
        dims, hidden, weight, targets = _loss_call(hidden, weight, targets)
        for name, t in (("lse", lse), ("row_weight", row_weight)):
            if t is not None and (t.dtype != torch.float32 or t.shape != (dims.N,) or not t.is_contiguous()):
                raise ValueError(f"{name} is {t.dtype} {tuple(t.shape)}: contiguous float32 ({dims.N},) is wanted")
        _on_device(lse=lse, row_weight=row_weight, hidden_grad=hidden_grad, weight_grad=weight_grad)
        if accumulate and weight_grad is None:
            raise ValueError("accumulate needs a weight_grad to add to")
        if hidden_grad is None and need[0]:
            hidden_grad = torch.empty((dims.N, dims.D), dtype=hidden.dtype, device=hidden.device)
        if weight_grad is None and need[1]:
            weight_grad = torch.empty((dims.V, dims.D), dtype=hidden.dtype, device=hidden.device)
        if hidden_grad is not None:
            hidden_grad, dims.hidden_grad_stride = _result(hidden_grad, "hidden_grad", (dims.N, dims.D), hidden.dtype)
        if weight_grad is not None:
            weight_grad, dims.weight_grad_stride = _result(weight_grad, "weight_grad", (dims.V, dims.D), hidden.dtype)
        if accumulate:
            dims.flags |= _px.PX_FLAG_ACCUMULATE
        workspace = _loss_scratch(dims, 1, workspace, hidden.device)
        _check(_px.lib().pollux_token_loss_grad(ctypes.byref(dims), hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), lse.data_ptr(),
                                                _px._ptr(row_weight), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                                _px._ptr(hidden_grad), _px._ptr(weight_grad), _px._stream_handle(stream)),
               "pollux_token_loss_grad")
    return hidden_grad, weight_grad
