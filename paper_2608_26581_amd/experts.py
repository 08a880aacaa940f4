"""Binding of the calls around a layer of experts: the router's choice, tokens
sorted by expert and back, and the product with a weight matrix per expert.

Each function carries the name of the C entry point it calls and checks its
tensors as the other calls do.  A plan is an ExpertPlan, or any three tensors of its
layout.  The router's weights are differentiable in the logits, gather in x and
combine in z and the weights, in reverse mode (a tangent of the forward mode is an
error); what goes through the 4-bit product is not.  A backward pass is captured into a
graph as torch has it for any: after a pass on a side stream, and with no eager graph of the
same leaves left alive.
"""
import ctypes
import threading
from typing import NamedTuple

import torch
from torch.autograd.forward_ad import unpack_dual
from torch.autograd.function import once_differentiable

from . import rfq as _binding
from .rfq import (
    _FLOAT, _OUT_CODE, _U8, _check, _dtype_code, _empty, _need, _need_pair, _ptr, _result, _stream,
    _torch_stream, _wants_grad, _written, _z_out, load,
)

_I32 = (torch.int32,)
_F32 = (torch.float32,)

# The entry points that the native calls use here, in the order their bind_experts() takes,
# and the module that has them.
_NATIVE_ENTRIES = (
    "rfq_route", "rfq_route_backward", "rfq_expert_sort", "rfq_expert_sort_workspace_bytes",
    "rfq_expert_gather", "rfq_expert_combine", "rfq_expert_combine_backward", "rfq_gemm_experts",
)
_bound = None
_bind_lock = threading.Lock()


def _native(func, *args):
    """The result of a native call, or None where the Python path takes over."""
    global _bound
    calls = _binding._calls
    if calls is None or _bound is not calls:
        lib = load()
        calls = _binding._calls
        if not calls:
            return None
        with _bind_lock:
            if _bound is not calls:
                calls.bind_experts(*(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value
                                     for f in _NATIVE_ENTRIES))
                _bound = calls
    return _result(func, getattr(calls, func)(*args))


class ExpertPlan(NamedTuple):
    """Where the pairs (token, choice) stand when sorted by expert (int32): the slots of
    expert e are offsets[e] .. offsets[e + 1] - 1 (offsets [E + 1]); rows [T k] is the token of
    each slot (-1 past the last), slots [T][k] the slot of each pair (-1: dropped)."""
    offsets: torch.Tensor
    rows: torch.Tensor
    slots: torch.Tensor


def _need_2d(t, name, dtypes, dev=None):
    _need(t, name, dtypes, None, dev)
    if t.dim() != 2:
        raise ValueError("%s must be 2-D" % name)


def _need_plan(plan, dev):
    """(rows, slots) of a plan, checked against each other."""
    offsets, rows, slots = plan
    _need(offsets, "offsets", _I32, None, dev)
    _need_2d(slots, "slots", _I32, dev)
    _need(rows, "rows", _I32, (slots.numel(),), dev)
    return rows, slots


def _apply(function, stream, device, *args):
    """A differentiable call on `stream` (autograd runs the gradient on the stream that
    is current here)."""
    if stream is None:
        return function.apply(*args)
    with torch.cuda.stream(_torch_stream(stream, device)):
        r = function.apply(*args)
    for t in r if isinstance(r, tuple) else (r,):
        t.record_stream(torch.cuda.current_stream(device))
    return r


def _dense(t):
    """A gradient as the calls take it: contiguous and 16-byte aligned."""
    return t if t.is_contiguous() and t.data_ptr() % 16 == 0 else t.clone(
        memory_format=torch.contiguous_format)


def _no_tangent(grad):
    """Refuses a gradient with a tangent where the backward pass is differentiable in neither
    mode (reverse mode is refused by once_differentiable)."""
    if unpack_dual(grad).tangent is not None:
        raise NotImplementedError("a backward pass of the calls around a layer of experts has no "
                                  "jvp: its gradient must not have a tangent of the forward mode")


# ---- the router

class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, renormalize):
        weights, experts = rfq_route(logits, k, renormalize)
        ctx.mark_non_differentiable(experts)
        ctx.save_for_backward(logits, weights, experts)
        ctx.renormalize = renormalize
        return weights, experts

    @staticmethod
    @once_differentiable
    def backward(ctx, dweights, _):
        _no_tangent(dweights)
        logits, weights, experts = ctx.saved_tensors
        return rfq_route_backward(_dense(dweights), logits, weights, experts,
                                  ctx.renormalize), None, None


def _route(logits, k, renormalize, stream):
    _need_2d(logits, "logits", _FLOAT)
    dev, (T, E) = logits.get_device(), logits.shape
    k = int(k)
    if not 1 <= k <= min(E, 16):
        raise ValueError("k must be 1 .. %d, not %d" % (min(E, 16), k))
    weights = _empty((T, k), torch.float32, logits.device, stream)
    experts = _empty((T, k), torch.int32, logits.device, stream)
    st = load().rfq_route(_ptr(logits), _dtype_code(logits), T, E, k, bool(renormalize),
                          _ptr(weights), _ptr(experts), _stream(stream, dev))
    _check("rfq_route", st)
    return weights, experts


def rfq_route(logits, k, renormalize=True, stream=None):
    """The k largest of logits [T][E] (bf16 or fp32) per token, ties to the lower index ->
    (weights [T][k] fp32, experts [T][k] int32): softmax over the chosen logits, or with
    renormalize False over all.  -inf is not chosen: expert -1, weight 0.  weights are
    differentiable in logits.  The two may be parts of one allocation (clone one that is to be
    resized, or saved by itself)."""
    if stream is None:
        r = _native("route", logits, k, renormalize)
        if r is not None:
            return r
    if _wants_grad(logits):
        return _apply(_Route, stream, logits.device, logits, k, renormalize)
    return _route(logits, k, renormalize, stream)


def rfq_route_backward(dweights, logits, weights, experts, renormalize=True, stream=None):
    """The gradient [T][E] (dtype of logits) of rfq_route(logits, k) -> weights, experts from
    that of its weights."""
    if stream is None:
        r = _native("route_backward", dweights, logits, weights, experts, renormalize)
        if r is not None:
            return r
    _need_2d(logits, "logits", _FLOAT)
    dev, (T, E) = logits.get_device(), logits.shape
    _need_2d(weights, "weights", _F32, dev)
    k = weights.shape[1]
    _need(weights, "weights", _F32, (T, k), dev)
    _need(dweights, "dweights", _F32, (T, k), dev)
    _need(experts, "experts", _I32, (T, k), dev)
    out = _empty((T, E), logits.dtype, logits.device, stream)
    st = load().rfq_route_backward(_ptr(dweights), _ptr(logits), _dtype_code(logits), T, E, k,
                                   _ptr(weights), _ptr(experts), bool(renormalize), _ptr(out),
                                   _stream(stream, dev))
    _check("rfq_route_backward", st)
    return out


# ---- the sort

def rfq_expert_sort_workspace_bytes(T, k, E):
    """Workspace of rfq_expert_sort for these sizes (0: one workgroup sorts)."""
    return int(load().rfq_expert_sort_workspace_bytes(int(T), int(k), int(E)))


def rfq_expert_sort(experts, n_experts, first=0, workspace=None, stream=None):
    """The pairs of experts [T][k] sorted by expert, those of an expert in their order ->
    ExpertPlan.  Experts outside [first, first + n_experts) are dropped.  workspace: a
    contiguous uint8 tensor of rfq_expert_sort_workspace_bytes, or None: one from torch's
    allocator.  The three may be parts of one allocation (clone one that is to be
    resized, or saved by itself)."""
    if stream is None:
        r = _native("expert_sort", experts, n_experts, first, workspace)
        if r is not None:
            return ExpertPlan(*r)
    _need_2d(experts, "experts", _I32)
    dev, (T, k) = experts.get_device(), experts.shape
    E = int(n_experts)
    if not 1 <= E <= 1024:
        raise ValueError("n_experts must be 1 .. 1024, not %d" % E)
    offsets, rows = (_empty(n, torch.int32, experts.device, stream) for n in (E + 1, T * k))
    slots = _empty((T, k), torch.int32, experts.device, stream)
    if workspace is None:
        nbytes = load().rfq_expert_sort_workspace_bytes(T, k, E)
        if nbytes > 0:
            workspace = _empty(nbytes, torch.uint8, experts.device, stream, returned=False)
    else:
        _need(workspace, "workspace", _U8, None, dev)
        nbytes = workspace.numel()
    st = load().rfq_expert_sort(_ptr(experts), T, k, int(first), E, _ptr(offsets), _ptr(rows),
                                _ptr(slots), _ptr(workspace), nbytes, _stream(stream, dev))
    _check("rfq_expert_sort", st)
    return ExpertPlan(offsets, rows, slots)


# ---- rows to the experts and back

class _Gather(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, offsets, rows, slots):
        ctx.save_for_backward(offsets, rows, slots)
        return rfq_expert_gather(x, (offsets, rows, slots))

    @staticmethod
    def backward(ctx, dxs):
        return rfq_expert_combine(_dense(dxs), None, ctx.saved_tensors), None, None, None


def _gather(x, plan, out, stream):
    _need_2d(x, "x", _FLOAT)
    dev, (T, N) = x.get_device(), x.shape
    rows, slots = _need_plan(plan, dev)
    if slots.shape[0] != T:
        raise ValueError("x has %d rows, the plan %d tokens" % (T, slots.shape[0]))
    P, given = rows.shape[0], out
    if out is None:
        out = _empty((P, N), x.dtype, x.device, stream)
    else:
        _need(out, "out", (x.dtype,), (P, N), dev)
    st = load().rfq_expert_gather(_ptr(x), _dtype_code(x), T, N, _ptr(rows), _ptr(slots),
                                  slots.shape[1], P, _ptr(out), _stream(stream, dev))
    _check("rfq_expert_gather", st)
    return out if given is None else _written(out)


def rfq_expert_gather(x, plan, out=None, stream=None):
    """xs [T k][N]: the rows of x [T][N] (bf16 or fp32) in the slots of the plan, zeros past the
    last.  Differentiable in x, without out."""
    if stream is None:
        r = _native("expert_gather", x, *plan, out)
        if r is not None:
            return r if out is None else _written(out)
    if _wants_grad(x, out):
        if out is not None:
            raise ValueError("out takes no gradient: x and out must not require one")
        return _apply(_Gather, stream, x.device, x, *plan)
    return _gather(x, plan, out, stream)


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, z, weights, offsets, rows, slots):
        ctx.save_for_backward(z, weights, offsets, rows, slots)
        return rfq_expert_combine(z, weights, (offsets, rows, slots))

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        _no_tangent(dout)
        z, weights, *plan = ctx.saved_tensors
        need_z, need_w = ctx.needs_input_grad[:2]
        dz, dw = _combine_backward(_dense(dout), z, weights, plan, need_z, need_w, None)
        return dz, dw, None, None, None


class _Sum(torch.autograd.Function):
    """combine without weights, the gradient of gather and gather's own gradient."""

    @staticmethod
    def forward(ctx, z, offsets, rows, slots):
        ctx.save_for_backward(offsets, rows, slots)
        return rfq_expert_combine(z, None, (offsets, rows, slots))

    @staticmethod
    def backward(ctx, dout):
        return rfq_expert_gather(_dense(dout), ctx.saved_tensors), None, None, None


def _combine(z, weights, plan, out, stream):
    _need_2d(z, "z", _FLOAT)
    dev, (P, N) = z.get_device(), z.shape
    rows, slots = _need_plan(plan, dev)
    T, k = slots.shape
    if rows.shape[0] != P:
        raise ValueError("z has %d rows, the plan %d slots" % (P, rows.shape[0]))
    if weights is not None:
        _need(weights, "weights", _F32, (T, k), dev)
    given = out
    if out is None:
        out = _empty((T, N), z.dtype, z.device, stream)
    else:
        _need(out, "out", (z.dtype,), (T, N), dev)
    st = load().rfq_expert_combine(_ptr(z), _dtype_code(z), P, N, _ptr(slots), _ptr(weights), T, k,
                                   _ptr(out), _stream(stream, dev))
    _check("rfq_expert_combine", st)
    return out if given is None else _written(out)


def rfq_expert_combine(z, weights, plan, out=None, stream=None):
    """out [T][N]: the sum over a token's choices of its weight (fp32 [T][k]; None: 1) times
    the row of z [T k][N] (bf16 or fp32) in the choice's slot; dropped choices add nothing.
    Differentiable in z and weights, without out."""
    if stream is None:
        r = _native("expert_combine", z, weights, *plan, out)
        if r is not None:
            return r if out is None else _written(out)
    if _wants_grad(z, weights, out):
        if out is not None:
            raise ValueError("out takes no gradient: z, weights and out must not require one")
        if weights is None:
            return _apply(_Sum, stream, z.device, z, *plan)
        return _apply(_Combine, stream, z.device, z, weights, *plan)
    return _combine(z, weights, plan, out, stream)


def _combine_backward(dout, z, weights, plan, need_z, need_w, stream):
    if stream is None and need_z and need_w:
        r = _native("expert_combine_backward", dout, z, weights, *plan)
        if r is not None:
            return r
    _need_2d(z, "z", _FLOAT)
    dev, (P, N) = z.get_device(), z.shape
    rows, slots = _need_plan(plan, dev)
    T, k = slots.shape
    if rows.shape[0] != P:
        raise ValueError("z has %d rows, the plan %d slots" % (P, rows.shape[0]))
    _need(dout, "dout", (z.dtype,), (T, N), dev)
    if weights is not None:
        _need(weights, "weights", _F32, (T, k), dev)
    dz = _empty((P, N), z.dtype, z.device, stream) if need_z else None
    dw = _empty((T, k), torch.float32, z.device, stream) if need_w else None
    st = load().rfq_expert_combine_backward(_ptr(dout), _ptr(z), _dtype_code(z), P, N, _ptr(rows),
                                            _ptr(slots), _ptr(weights), T, k, _ptr(dz), _ptr(dw),
                                            _stream(stream, dev))
    _check("rfq_expert_combine_backward", st)
    return dz, dw


def rfq_expert_combine_backward(dout, z, weights, plan, stream=None):
    """(dz, dweights): the gradients of rfq_expert_combine(z, weights, plan) from that of its
    result; rows of dz that no pair names are zeros."""
    return _combine_backward(dout, z, weights, plan, True, True, stream)


# ---- the product

def rfq_gemm_experts(q_codes, q_scales, r_codes, r_scales, w_codes, w_scales, offsets, rows=None,
                     out_dtype=torch.float32, out=None, stream=None):
    """Z[P][N]: slot s of expert e (offsets[e] <= s < offsets[e + 1]) is activation row rows[s]
    (rows None: row s) times w_codes [E][N][K/2], w_scales [E][N][K/32]; r_* None gives plain
    MXFP4.  Rows of Z that belong to no expert are not written; a row index outside the
    activations counts as a row of zeros."""
    if stream is None:
        r = _native("gemm_experts", q_codes, q_scales, r_codes, r_scales, w_codes, w_scales, offsets,
                    rows, _OUT_CODE.get(out_dtype, 2), out)
        if r is not None:
            return r if out is None else _written(out)
    _need_2d(q_codes, "q codes", _U8)
    dev, M, K = q_codes.get_device(), q_codes.shape[0], 2 * q_codes.shape[1]
    _need(q_scales, "q scales", _U8, (M, K // 32), dev)
    _need_pair(r_codes, r_scales, M, K, "r", dev)
    _need(w_codes, "w codes", _U8, None, dev)
    if w_codes.dim() != 3:
        raise ValueError("w codes must be 3-D [E][N][K/2]")
    E, N = w_codes.shape[:2]
    _need(w_codes, "w codes", _U8, (E, N, K // 2), dev)
    _need(w_scales, "w scales", _U8, (E, N, K // 32), dev)
    _need(offsets, "offsets", _I32, (E + 1,), dev)
    P = M
    if rows is not None:
        _need(rows, "rows", _I32, None, dev)
        if rows.dim() != 1:
            raise ValueError("rows must be 1-D [P]")
        P = rows.shape[0]
    z = _z_out(out, out_dtype, P, N, q_codes.device, stream, dev)
    st = load().rfq_gemm_experts(_ptr(q_codes), _ptr(q_scales), _ptr(r_codes), _ptr(r_scales),
                                 _ptr(w_codes), _ptr(w_scales), _ptr(offsets), _ptr(rows), M, P, E,
                                 N, K, _ptr(z), _dtype_code(z), _stream(stream, dev))
    _check("rfq_gemm_experts", st)
    return z if out is None else _written(z)
