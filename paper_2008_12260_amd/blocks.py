"""The operators of a residual block on torch device tensors (C ABI in include/pollux.h, "A residual block of a language-model job"): the
edges between a job's blocks, its gated activations, and what of them is remembered for the backward pass in 8 bits.

One block, its products a job's own:

    rows          the last edge's
    gate, up      products of rows
    a, *kept      gated(gate, up, keep="i8")
    branch        a product of a
    y, rows, s    block_edge(y, branch, gate=..., after=Norm(...), before=Norm(...), keep="i8")

and backward from block_edge_grad(...), through gated_grad(da, *kept), to kept_grad(s.y_kept, ...), the gradient of the weights that rows met.

As in train.py, arguments are checked and marshalled here, results are allocated by torch on the stream that the call is enqueued on, nothing synchronises or
records for autograd, and a tensor that requires grad is refused where grad mode is on, one with a forward-mode tangent anywhere.
"""
from __future__ import annotations

import ctypes
import functools
import math
from typing import NamedTuple, Optional

import paper_2008_12260_amd as _px

from .train import _check, _contiguous, _no_tangents, _on, _on_device, _planned, _scratch, _type

_FORMS = {None: _px.PX_KEPT_NONE, "i8": _px.PX_KEPT_I8, "e4m3": _px.PX_KEPT_E4M3}
_ACTS = {"silu": _px.PX_ACT_SILU, "gelu": _px.PX_ACT_GELU, "gelu_tanh": _px.PX_ACT_GELU_TANH}
_GROUP = 32


class Kept(NamedTuple):
    """N rows of `width` elements in 8 bits: values [N, W] (W: width in whole groups of 32) and scales [N, W / 32], uint8; form "i8" or "e4m3"."""
    values: "torch.Tensor"
    scales: "torch.Tensor"
    width: int
    form: str


class Norm(NamedTuple):
    """A norm's weights and biases [D]; None: 1 and 0."""
    weight: Optional["torch.Tensor"] = None
    bias: Optional["torch.Tensor"] = None


class EdgeState(NamedTuple):
    """What block_edge leaves for block_edge_grad: (mean, 1 / spread) of each norm's rows [N, 2], the normalised rows where they are kept, the types of x and of
    the branch, and whether there was one."""
    y_stats: Optional["torch.Tensor"]
    branch_stats: Optional["torch.Tensor"]
    y_kept: Optional[Kept]
    branch_kept: Optional[Kept]
    x_dtype: "torch.dtype"
    dtype: "torch.dtype"
    branched: bool


class EdgeGrads(NamedTuple):
    x: Optional["torch.Tensor"]
    branch: Optional["torch.Tensor"]
    gate: Optional["torch.Tensor"]
    after_weight: Optional["torch.Tensor"]
    after_bias: Optional["torch.Tensor"]
    before_weight: Optional["torch.Tensor"]
    before_bias: Optional["torch.Tensor"]


@functools.lru_cache(maxsize=1024)
def _dims(cls, signs, *values):
    """The library's description of a call that takes no scratch memory; signs: of the values that may be zeros of either sign."""
    return ctypes.byref(cls(*values))


def _form(form):
    if form not in _FORMS:
        raise ValueError(f"form is {form!r}: 'i8' or 'e4m3' is wanted")
    return _FORMS[form]


def _matrix(t, name, most=(1 << 20) - 1):
    """(the tensor as rows, their stride): [..., D] as [N, D], as it is where rows are contiguous, one after the other or at most `most` apart, else copied."""
    if t.dim() == 0:
        raise ValueError(f"{name} has no dimensions: rows are wanted")
    D = t.shape[-1]
    if t.dim() != 2:
        t = t.reshape(-1, D) if D else t.reshape(math.prod(t.shape[:-1]), 0)
    ld, step = t.stride()
    if D > 1 and step != 1 or t.shape[0] > 1 and ld != D and not D < ld <= most:
        t, ld = t.clone(memory_format=_contiguous()), D
    return t, ld if t.shape[0] > 1 else D


def _written(t, name, shape, dtype):
    """(a caller's result as rows, their stride)"""
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype} {tuple(t.shape)}: {dtype} {tuple(shape)} is wanted")
    D = shape[-1]
    try:
        rows = t.view(-1, D) if t.dim() != 2 else t
    except RuntimeError:
        rows = None
    if rows is None or D > 1 and rows.stride(1) != 1 or rows.shape[0] > 1 and rows.stride(0) != D and not D < rows.stride(0) < 1 << 20:
        raise ValueError(f"{name} needs contiguous rows, one stride apart")
    return rows, rows.stride(0) if rows.shape[0] > 1 else D


def _kept(k, name, rows=None, width=None):
    """The Kept as the library takes it."""
    import torch
    values, scales, D, form = k
    W = -(-D // _GROUP) * _GROUP
    if D < 1 or values.dtype != torch.uint8 or scales.dtype != torch.uint8 or values.dim() != 2 or values.shape[1] != W or scales.shape != (values.shape[0], W // _GROUP):
        raise ValueError(f"{name} has values {values.dtype} {tuple(values.shape)} and scales {scales.dtype} {tuple(scales.shape)}: uint8 [N, {W}] and [N, {W // _GROUP}] are wanted")
    if rows is not None and values.shape[0] != rows or width is not None and D != width:
        raise ValueError(f"{name} has {values.shape[0]} rows of {D} elements: {values.shape[0] if rows is None else rows} of {D if width is None else width} are wanted")
    if form is None:
        raise ValueError("form is None: 'i8' or 'e4m3' is wanted")
    _form(form)
    _on_device(values, scales)
    values, scales = values.contiguous(), scales.contiguous()
    if values.data_ptr() & 15:
        values = values.clone()
    return Kept(values, scales, D, form)


def _new_kept(rows, D, form):
    """Of rows on the same device."""
    import torch
    N, W = rows.shape[0], -(-D // _GROUP) * _GROUP
    return Kept(rows.new_empty((N, W), dtype=torch.uint8), rows.new_empty((N, W // _GROUP), dtype=torch.uint8), D, form)


# New tensors are asked of one that is there: a microsecond less than torch.empty with the same attributes.
def _like(t):
    """Contiguous, of t's shape and type."""
    import torch
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _vectors(D, **named):
    """(their one type, the tensors): vectors of D elements, or None."""
    dtype, out = None, []
    for name, t in named.items():
        if t is not None:
            if t.shape != (D,):
                raise ValueError(f"{name} has shape {tuple(t.shape)}: ({D},) is wanted")
            if dtype is not None and t.dtype != dtype:
                raise TypeError(f"{name} is {t.dtype} and another weight {dtype}: one type is wanted")
            dtype = t.dtype
            t = t.contiguous()
        out.append(t)
    return dtype, out


def keep(rows, form="i8", stream=None):
    """rows [..., D] in 8 bits, as [N, D]: 32 neighbours of a row share a power of two; form "i8" (within 1/127 of the largest of the 32) or "e4m3" (within 2^-4 of
    the element).  Groups that hold an infinity or a NaN are restored as NaN; sizes next to 2^128 (from 1.984 * 2^127 on, and 1.9375 * 2^127) round to it and are restored as infinite."""
    _untracked_here(rows)
    with _on(stream):
        _on_device(rows)
        type_, code = _type(rows, "rows"), _form(form)
        if code == _px.PX_KEPT_NONE:
            raise ValueError("form is None: 'i8' or 'e4m3' is wanted")
        rows, ld = _matrix(rows, "rows")
        N, D = rows.shape
        kept = _new_kept(rows, D, form)
        _check(_px.lib().pollux_keep(_dims(_px.KeepDims, None, N, D, type_, code, 0, ld), rows.data_ptr(), kept.values.data_ptr(), kept.scales.data_ptr(),
                                     _px._stream_handle(stream)), "pollux_keep")
    return kept


def restore(kept, dtype=None, out=None, stream=None):
    """The rows [N, D] that `kept` stands for, in `dtype` (None: bfloat16, which holds them exactly), or in `out`."""
    import torch
    _untracked_here(out)
    with _on(stream):
        _on_device(out)
        kept = _kept(kept, "kept")
        N, D = kept.values.shape[0], kept.width
        if out is None:
            out = kept.values.new_empty((N, D), dtype=torch.bfloat16 if dtype is None else dtype)
        rows, ld = _written(out, "out", (N, D), out.dtype if dtype is None else dtype)
        _check(_px.lib().pollux_restore(_dims(_px.KeepDims, None, N, D, _type(rows, "rows"), _form(kept.form), 0, ld), kept.values.data_ptr(), kept.scales.data_ptr(),
                                        rows.data_ptr(), _px._stream_handle(stream)), "pollux_restore")
    return out


def _untracked_here(*tensors):
    import torch
    _no_tangents(torch, tensors)
    if not torch.is_grad_enabled():
        return
    for t in tensors:
        if t is not None and t.requires_grad:
            raise ValueError(f"a tensor {tuple(t.shape)} requires grad, which this call does not record: detach it, or call under torch.no_grad(), "
                             "and take the gradients from block_edge_grad, gated_grad and kept_grad")


def kept_grad(kept, rows_grad, weight=None, bias=None, weight_grad=None, accumulate=False, workspace=None, stream=None):
    """The gradient [M, D] of a layer's weights from its input, kept [N, D], and the gradient of its result, rows_grad [..., M] as [N, M], in the latter's type:
    rows_grad' (kept * weight + bias).  weight, bias [D]: of the norm whose rows are kept, where the layer's input was those times weight, plus bias.  accumulate: weight_grad is given and added to."""
    import torch
    _untracked_here(rows_grad, weight, bias, weight_grad)
    with _on(stream):
        _on_device(rows_grad, weight, bias, weight_grad)
        type_ = _type(rows_grad, "rows_grad")
        rows, ld = _matrix(rows_grad, "rows_grad")
        if rows.data_ptr() & 15:
            rows, ld = rows.clone(memory_format=_contiguous()), rows.shape[1]
        N, M = rows.shape
        kept = _kept(kept, "kept", rows=N)
        D = kept.width
        dtype, (weight, bias) = _vectors(D, weight=weight, bias=bias)
        weight_type = type_ if dtype is None else _type(bias if weight is None else weight, "weight")
        if accumulate and weight_grad is None:
            raise ValueError("accumulate needs a weight_grad to add to")
        if weight_grad is None:
            weight_grad = rows.new_empty((M, D))
        out, out_ld = _written(weight_grad, "weight_grad", (M, D), rows.dtype)
        if out.data_ptr() & 15:
            raise ValueError("weight_grad needs a base aligned to 16 bytes")
        dims, need = _planned(_px.KeptGradDims, "pollux_kept_grad_workspace_size", (), None, N, D, M, type_, weight_type, _form(kept.form),
                              _px.PX_FLAG_ACCUMULATE if accumulate else 0, ld, out_ld)
        workspace, size = _scratch(workspace, need, rows.device)
        _check(_px.lib().pollux_kept_grad(dims, kept.values.data_ptr(), kept.scales.data_ptr(), rows.data_ptr(), _px._ptr(weight), _px._ptr(bias), workspace.data_ptr(), size,
                                          out.data_ptr(), _px._stream_handle(stream)), "pollux_kept_grad")
    return weight_grad


def _gate(gate, shape, N, D):
    """(the gate as rows, of how many rows of [*shape] each serves: 0 for one that serves all)"""
    if gate is None:
        return None, 0
    if gate.dim() == 0 or gate.shape[-1] != D:
        raise ValueError(f"gate has shape {tuple(gate.shape)}: rows of {D} are wanted")
    if gate.dim() == 1:
        return gate.contiguous(), 0
    lead = tuple(gate.shape[:-1])
    if gate.dim() <= len(shape) > 2:
        # What broadcasts over a dimension before one that it has serves rows that are not neighbours.  Of fewer dimensions it is one of x's first ones, or one that broadcasts to no other rows.
        at = (1,) * (len(shape) - gate.dim()) + lead
        k = next((k for k in range(len(shape) - 1) if at[k] != shape[k]), len(shape) - 1)
        if any(size != 1 for size in at[k:]) and (len(at) == len(lead) or lead != tuple(shape[:len(lead)]) and all(a in (1, b) for a, b in zip(at, shape))):
            raise ValueError(f"gate has shape {tuple(gate.shape)} beside {tuple(shape)}: the first dimensions of that, and ones, are wanted")
    flat = gate.reshape(-1, D).contiguous()
    G = flat.shape[0]
    if G != 1 and (N % G if G else N):
        raise ValueError(f"a gate of {G} rows does not divide {N} rows")
    return flat, 0 if G == 1 else N // G if N else 1


def _zeros(*values):
    return tuple(math.copysign(1.0, v) for v in values)


def block_edge(x, branch=None, gate=None, after=None, before=None, residual=1.0, scale=1.0, eps=1e-6, centred=False, keep=None, rows_dtype=None, stream=None):
    """(y, rows, state): y = residual * x + scale * gate * after(branch), rows = before(y); all [..., D], in one pass.

    after, before: Norm, or None for no norm (`rows` is then None); centred: norms subtract the mean.  branch None: y is x, and the call is the norm `before`
    (residual and scale then count for nothing, here and in block_edge_grad: a stack may give all its edges the same).
    gate: [D], or [..., D] of G rows, each of which serves N / G rows in turn (one a sequence, [B, 1, D] or [B, D], one a token); one that would broadcast over other rows
    (one a position, [T, D] beside [B, T, D]) is refused.  x may be float32 beside a branch of 16 bits: y has x's type, rows the branch's
    (rows_dtype, or x's, without one).  keep "i8" or "e4m3": the normalised rows, which block_edge_grad needs, are left in 8 bits in `state`, and y and branch need not be remembered."""
    import torch
    weights = (*(after or ()), *(before or ()))
    _untracked_here(x, branch, gate, *weights)
    with _on(stream):
        _on_device(x, branch, gate, *weights)
        x_type, form = _type(x, "x"), _form(keep)
        if branch is None and (after is not None or gate is not None or before is None):
            raise ValueError("without a branch there is a norm `before`, and neither gate nor norm `after`")
        if branch is not None and (branch.shape != x.shape or rows_dtype is not None and rows_dtype != branch.dtype):
            raise ValueError(f"branch is {branch.dtype} {tuple(branch.shape)} beside x {tuple(x.shape)}: one shape, and rows of the branch's type, are wanted")
        shape, dtype = x.shape, (x.dtype if rows_dtype is None else rows_dtype) if branch is None else branch.dtype
        x_rows, x_ld = _matrix(x, "x")
        N, D = x_rows.shape
        branch_rows, branch_ld = (None, 0) if branch is None else _matrix(branch, "branch")
        gate_rows, span = _gate(gate, shape, N, D)
        weight_dtype, (w_a, b_a, w_b, b_b) = _vectors(D, after_weight=after and after[0], after_bias=after and after[1], before_weight=before and before[0],
                                                      before_bias=before and before[1])
        y = x if branch is None else _like(x)
        rows = None if before is None else _like(branch) if branch is not None else x.new_empty(shape, dtype=dtype)
        branch_stats = None if after is None else x.new_empty((N, 2), dtype=torch.float32)
        y_stats = None if before is None else x.new_empty((N, 2), dtype=torch.float32)
        branch_kept = _new_kept(x_rows, D, keep) if form and (after is not None or gate is not None) else None
        y_kept = _new_kept(x_rows, D, keep) if form and before is not None else None
        flags = (_px.PX_EDGE_AFTER if after is not None else 0) | (_px.PX_EDGE_BEFORE if before is not None else 0) | (_px.PX_EDGE_CENTRED if centred else 0)
        eps, residual, scale = float(eps), 1.0 if branch is None else float(residual), float(scale)
        dims = _dims(_px.EdgeDims, _zeros(eps, residual, scale), N, D, x_type, _type_of(dtype), _type_of(weight_dtype), _type_of(gate_rows.dtype if gate_rows is not None else None), form, flags,
                     eps, residual, scale, span, x_ld, branch_ld, 0, 0, 0, 0, 0, 0)
        ptr = _px._ptr
        _check(_px.lib().pollux_block_edge(dims, x_rows.data_ptr(), ptr(branch_rows), ptr(gate_rows), ptr(w_a), ptr(b_a), ptr(w_b), ptr(b_b),
                                           None if branch is None else y.data_ptr(), ptr(rows), ptr(y_stats), ptr(branch_stats),
                                           *((None, None) if y_kept is None else (y_kept.values.data_ptr(), y_kept.scales.data_ptr())),
                                           *((None, None) if branch_kept is None else (branch_kept.values.data_ptr(), branch_kept.scales.data_ptr())),
                                           _px._stream_handle(stream)), "pollux_block_edge")
    return y, rows, EdgeState(y_stats, branch_stats, y_kept, branch_kept, x.dtype, dtype, branch is not None)


_TYPES = {}


def _type_of(dtype):
    """A type's code; of none, fp32's."""
    if not _TYPES:
        import torch
        _TYPES.update({None: _px.PX_TYPE_F32, torch.float32: _px.PX_TYPE_F32, torch.bfloat16: _px.PX_TYPE_BF16, torch.float16: _px.PX_TYPE_F16})
    if dtype not in _TYPES:
        raise TypeError(f"{dtype}: float32, bfloat16 or float16 is wanted")
    return _TYPES[dtype]


def _stats(t, name, N):
    import torch
    if t is None or t.dtype != torch.float32 or t.shape != (N, 2) or not t.is_contiguous():
        raise ValueError(f"state has no {name} of {N} rows")
    return t


_ALL = ("x", "branch", "gate", "after", "before")


def block_edge_grad(y_grad, rows_grad, state, y=None, branch=None, gate=None, after=None, before=None, residual=1.0, scale=1.0, centred=False, need=_ALL, workspace=None,
                    stream=None):
    """EdgeGrads of block_edge: the gradients of x, branch, gate and of the norms' weights and biases, from those of y (None: zeros) and of rows.

    gate, after, before, residual, scale, centred: as in the call that left `state`.  Where it kept nothing, y and branch are given as that call returned and
    took them (a branch without norm and gate need not be).  need: what is wanted of the gradients; None stands in the place of the others."""
    import torch
    weights = (*(after or ()), *(before or ()))
    _untracked_here(y_grad, rows_grad, y, branch, gate, *weights)
    with _on(stream):
        kept = state.y_kept if state.y_kept is not None else state.branch_kept
        _on_device(y_grad, rows_grad, y, branch, gate, state.y_stats, state.branch_stats, *weights)
        if (before is None) != (state.y_stats is None) or (after is None) != (state.branch_stats is None) or not state.branched and (after is not None or gate is not None):
            raise ValueError("state is of a call with other norms or another branch")
        if (rows_grad is None) != (before is None):
            raise ValueError("rows_grad is given where there is a norm `before`, and only there")
        model = y_grad if y_grad is not None else rows_grad
        if model is None:
            raise ValueError("one of y_grad and rows_grad is wanted")
        shape = model.shape
        for name, t, dtype in (("y_grad", y_grad, state.x_dtype), ("rows_grad", rows_grad, state.dtype)):
            if t is not None and (t.shape != shape or t.dtype != dtype):
                raise ValueError(f"{name} is {t.dtype} {tuple(t.shape)}: {dtype} {tuple(shape)} is wanted")
        y_grad_rows, y_grad_ld = (None, 0) if y_grad is None else _matrix(y_grad, "y_grad")
        rows_grad_rows, rows_grad_ld = (None, 0) if rows_grad is None else _matrix(rows_grad, "rows_grad")
        N, D = (rows_grad_rows if y_grad_rows is None else y_grad_rows).shape
        device = model.device
        gate_rows, span = _gate(gate, shape, N, D)
        weight_dtype, (w_a, b_a, w_b, b_b) = _vectors(D, after_weight=after and after[0], after_bias=after and after[1], before_weight=before and before[0],
                                                      before_bias=before and before[1])
        if need is not _ALL and set(need) - set(_ALL):
            raise ValueError(f"need names {sorted(need)}: some of {_ALL} are wanted")

        def like(t, part):
            return None if t is None or part not in need else _like(t)
        x_grad = model.new_empty(shape, dtype=state.x_dtype) if "x" in need else None
        branch_grad = model.new_empty(shape, dtype=state.dtype) if state.branched and "branch" in need else None
        gate_grad = like(gate, "gate")
        if gate_grad is not None and N == 0 and span:
            gate_grad.zero_()                # of no rows the library knows no spans
        after_grads = like(w_a, "after"), like(b_a, "after")
        before_grads = like(w_b, "before"), like(b_b, "before")
        # what the norms were of: kept, or as it was
        asked = after is not None or gate_grad is not None
        y_rows = branch_rows = y_scales = branch_scales = None
        y_ld = branch_ld = 0
        form = _px.PX_KEPT_NONE
        if kept is not None:
            form = _form(kept.form)
            if any(k is not None and k.form != kept.form for k in (state.y_kept, state.branch_kept)) or before is not None and state.y_kept is None or asked and state.branch_kept is None:
                raise ValueError("state keeps not what is wanted of it, in one form")
            if before is not None:
                y_rows, y_scales = _kept(state.y_kept, "state.y_kept", N, D)[:2]
            if asked:
                branch_rows, branch_scales = _kept(state.branch_kept, "state.branch_kept", N, D)[:2]
        else:
            for name, t, dtype, there in (("y", y, state.x_dtype, before is not None), ("branch", branch, state.dtype, asked)):
                if there and (t is None or t.shape != shape or t.dtype != dtype):
                    raise ValueError(f"state keeps no rows: {name} is wanted, {dtype} {tuple(shape)}")
            if before is not None:
                y_rows, y_ld = _matrix(y, "y")
            if asked:
                branch_rows, branch_ld = _matrix(branch, "branch")
        if before is not None:
            _stats(state.y_stats, "y_stats", N)
        if after is not None:
            _stats(state.branch_stats, "branch_stats", N)
        flags = (_px.PX_EDGE_AFTER if after is not None else 0) | (_px.PX_EDGE_BEFORE if before is not None else 0) | (_px.PX_EDGE_CENTRED if centred else 0)
        residual, scale = float(residual) if state.branched else 1.0, float(scale)
        dims, bytes_ = _planned(_px.EdgeDims, "pollux_block_edge_workspace_size", (), _zeros(residual, scale), N, D, _type_of(state.x_dtype), _type_of(state.dtype), _type_of(weight_dtype),
                                _type_of(gate_rows.dtype if gate_rows is not None else None), form, flags, 0.0, residual, scale, span, 0, branch_ld, y_ld, 0, 0, 0,
                                y_grad_ld, rows_grad_ld)
        workspace, size = _scratch(workspace, bytes_, device)
        ptr = _px._ptr
        _check(_px.lib().pollux_block_edge_grad(dims, ptr(y_grad_rows), ptr(rows_grad_rows), ptr(y_rows), ptr(y_scales), ptr(branch_rows), ptr(branch_scales), ptr(state.y_stats),
                                                ptr(state.branch_stats), ptr(gate_rows), ptr(w_a), ptr(b_a), ptr(w_b), workspace.data_ptr(), size, ptr(x_grad), ptr(branch_grad),
                                                ptr(gate_grad), *map(ptr, after_grads), *map(ptr, before_grads), _px._stream_handle(stream)), "pollux_block_edge_grad")
    return EdgeGrads(x_grad, branch_grad, gate_grad, *after_grads, *before_grads)


def gated(gate, up=None, act="silu", keep=None, stream=None):
    """(rows, gate_kept, up_kept): rows = act(gate) * up (up None: act(gate)), all [..., F]; act "silu", "gelu" or "gelu_tanh".  keep "i8" or "e4m3": gate and up in
    8 bits, for gated_grad; else None in their places.  gate and up may be the halves of one product's rows."""
    import torch
    _untracked_here(gate, up)
    with _on(stream):
        _on_device(gate, up)
        type_, form = _type(gate, "gate"), _form(keep)
        if act not in _ACTS:
            raise ValueError(f"act is {act!r}: one of {', '.join(_ACTS)} is wanted")
        if up is not None and (up.shape != gate.shape or up.dtype != gate.dtype):
            raise ValueError(f"up is {up.dtype} {tuple(up.shape)}: {gate.dtype} {tuple(gate.shape)} is wanted")
        gate_rows, gate_ld = _matrix(gate, "gate", 1 << 20)
        up_rows, up_ld = (None, 0) if up is None else _matrix(up, "up", 1 << 20)
        N, F = gate_rows.shape
        rows = _like(gate)
        gate_kept = _new_kept(gate_rows, F, keep) if form else None
        up_kept = _new_kept(gate_rows, F, keep) if form and up is not None else None
        dims = _dims(_px.GatedDims, None, N, F, type_, _ACTS[act], form, 0, gate_ld, up_ld, 0, 0, 0, 0)
        ptr = _px._ptr
        _check(_px.lib().pollux_gated(dims, gate_rows.data_ptr(), ptr(up_rows), rows.data_ptr(), *((None, None) if gate_kept is None else map(ptr, gate_kept[:2])),
                                      *((None, None) if up_kept is None else map(ptr, up_kept[:2])), _px._stream_handle(stream)), "pollux_gated")
    return rows, gate_kept, up_kept


def gated_grad(rows_grad, gate, up=None, act="silu", want_rows=False, out=None, stream=None):
    """(gate_grad, up_grad, rows) of gated, from the gradient of its rows: gate and up as that call took them, or both as it kept them.

    The gradients are the halves of one tensor [..., 2 F] (`out`, where it is given; [..., F] without up): one product takes both.  want_rows: the rows again, formed from what is given here, else None."""
    import torch
    _untracked_here(rows_grad, None if isinstance(gate, Kept) else gate, None if isinstance(up, Kept) else up, out)
    with _on(stream):
        _on_device(rows_grad, None if isinstance(gate, Kept) else gate, None if isinstance(up, Kept) else up, out)
        type_ = _type(rows_grad, "rows_grad")
        if act not in _ACTS:
            raise ValueError(f"act is {act!r}: one of {', '.join(_ACTS)} is wanted")
        shape, dtype = rows_grad.shape, rows_grad.dtype
        d, d_ld = _matrix(rows_grad, "rows_grad")
        N, F = d.shape
        gate_scales = up_scales = None
        gate_ld = up_ld = 0
        form = _px.PX_KEPT_NONE
        if isinstance(gate, Kept):
            if up is not None and (not isinstance(up, Kept) or up.form != gate.form):
                raise ValueError("gate and up are both kept, in one form, or neither is")
            form = _form(gate.form)
            gate_rows, gate_scales = _kept(gate, "gate", N, F)[:2]
            up_rows, up_scales = (None, None) if up is None else _kept(up, "up", N, F)[:2]
        else:
            if isinstance(up, Kept):
                raise ValueError("gate and up are both kept, in one form, or neither is")
            for name, t in (("gate", gate), ("up", up)):
                if t is not None and (t.shape != shape or t.dtype != dtype):
                    raise ValueError(f"{name} is {t.dtype} {tuple(t.shape)}: {dtype} {tuple(shape)} is wanted")
            gate_rows, gate_ld = _matrix(gate, "gate", 1 << 20)
            up_rows, up_ld = (None, 0) if up is None else _matrix(up, "up", 1 << 20)
        halves = 1 if up is None else 2
        if out is None:
            out = d.new_empty((*shape[:-1], halves * F))
        both, ld = _written(out, "out", (*shape[:-1], halves * F), dtype)
        rows = _like(rows_grad) if want_rows else None
        dims = _dims(_px.GatedDims, None, N, F, type_, _ACTS[act], form, 0, gate_ld, up_ld, 0, d_ld, ld, ld)
        ptr = _px._ptr
        _check(_px.lib().pollux_gated_grad(dims, d.data_ptr(), gate_rows.data_ptr(), ptr(gate_scales), ptr(up_rows), ptr(up_scales), both.data_ptr(),
                                           None if up is None else both.data_ptr() + F * both.element_size(), ptr(rows), _px._stream_handle(stream)), "pollux_gated_grad")
    return (out, None, rows) if up is None else (out[..., :F], out[..., F:], rows)
