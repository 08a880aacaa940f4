"""Binding of the key/value cache calls: block tables, rotary positions, the
cache's write and read-back, and attention over the cache.

Each function carries the name of the C entry point it calls and checks its
tensors as the other calls do.  q, k, v and outputs are [T][H][D] device tensors
whose channels are contiguous; tokens and heads may be strided (slices of one
joint projection).  A cache is a KvCache, or any four tensors of its layout.
The rotation is differentiable; what goes through the 4-bit cache is not, and
results of those calls carry no gradient.
"""
import ctypes
import threading
from typing import NamedTuple

import torch

from . import rfq as _binding
from .rfq import (
    _FLOAT, _OUT_CODE, _U8, RFQ_BF16, RFQ_F32, Heads, KvCacheArgs, RopeSpec, _check, _dtype_code,
    _empty, _need, _ptr, _result, _stream, _torch_stream, _written, load,
)

_I32 = (torch.int32,)
_BF16 = (torch.bfloat16,)

# The entry points that the native calls use here, in the order their bind_kv()
# takes, and the module that has them.
_NATIVE_ENTRIES = (
    "rfq_block_assign", "rfq_block_release", "rfq_rope", "rfq_rope_backward", "rfq_kv_append",
    "rfq_kv_gather", "rfq_kv_attention", "rfq_kv_attention_workspace_bytes",
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
                calls.bind_kv(*(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value
                                for f in _NATIVE_ENTRIES))
                _bound = calls
    return _result(func, getattr(calls, func)(*args))


class KvCache(NamedTuple):
    """MXFP4 codes [blocks][heads][page][D / 2] and E8M0 scales
    [blocks][heads][page][D / 32] of a layer's keys and values (uint8)."""
    k_codes: torch.Tensor
    k_scales: torch.Tensor
    v_codes: torch.Tensor
    v_scales: torch.Tensor


def kv_cache(blocks, heads, page, D, device="cuda"):
    """An empty KvCache; nothing has to be initialised."""
    def part(width):
        return torch.empty((blocks, heads, page, width), dtype=torch.uint8, device=device)
    return KvCache(part(D // 2), part(D // 32), part(D // 2), part(D // 32))


def rope_table(max_pos, rotary, theta=10000.0, device="cuda"):
    """cos_sin [max_pos][rotary / 2][2] (fp32, rounded from 64 bits) of the angles
    p * theta ** (-2 j / rotary)."""
    freq = float(theta) ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)
    angle = torch.arange(max_pos, dtype=torch.float64)[:, None] * freq
    return torch.stack((torch.cos(angle), torch.sin(angle)), -1).float().contiguous().to(device)


def rope_axes(sections):
    """The axis of each rotated pair for contiguous sections of pairs, e.g.
    (16, 24, 24): 16 pairs turn by axis 0, 24 by axis 1, 24 by axis 2."""
    return b"".join(bytes([a]) * n for a, n in enumerate(sections))


def _need_heads(t, name, dtypes, shape=None, dev=None):
    """[T][H][D] with contiguous channels on the current device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    cur = torch.cuda.current_device() if dev is None else dev
    if t.get_device() != cur:
        raise ValueError("%s is on %s, not on the current device cuda:%d" % (name, t.device, cur))
    if t.dim() != 3:
        raise ValueError("%s must be 3-D [T][H][D]" % name)
    if t.dtype not in dtypes:
        raise TypeError("%s must be %s, not %s" % (name, " or ".join(map(str, dtypes)), t.dtype))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError("%s must have contiguous channels" % name)


def _heads(t):
    return Heads(t.data_ptr(), t.stride(0), t.stride(1))


def _rope(positions, cos_sin, axes, interleaved, T, dev):
    """The rfq_rope_spec of a call (keeps its host memory alive)."""
    if isinstance(positions, torch.Tensor) and positions.dim() == 1:
        positions = positions[None]
    if not isinstance(positions, torch.Tensor) or positions.dim() != 2:
        raise ValueError("positions must be a tensor [T] or [axes][T]")
    if not positions.is_cuda or positions.get_device() != dev:
        raise ValueError("positions must be on the current device cuda:%d" % dev)
    if positions.dtype != torch.int32:
        raise TypeError("positions must be torch.int32, not %s" % positions.dtype)
    if positions.shape[1] != T or (T > 1 and positions.stride(1) != 1):
        raise ValueError("positions must have one contiguous entry per token and axis")
    _need(cos_sin, "cos_sin", (torch.float32,), None, dev)
    if cos_sin.dim() != 3 or cos_sin.shape[2] != 2:
        raise ValueError("cos_sin must be [max_pos][rotary / 2][2]")
    half = cos_sin.shape[1]
    if axes is not None:
        axes = bytes(axes)
        if len(axes) != half:
            raise ValueError("axes must have one entry per rotated pair (%d), not %d"
                             % (half, len(axes)))
    spec = RopeSpec(positions.data_ptr(), positions.stride(0), cos_sin.data_ptr(),
                    cos_sin.shape[0], axes, positions.shape[0], 2 * half, bool(interleaved))
    return spec


def _need_cache(cache, dev):
    kc, ks, vc, vs = cache
    _need(kc, "k_codes", _U8, None, dev)
    if kc.dim() != 4:
        raise ValueError("k_codes must be 4-D [blocks][heads][page][D / 2]")
    blocks, heads, page, half = kc.shape
    _need(ks, "k_scales", _U8, (blocks, heads, page, half // 16), dev)
    _need(vc, "v_codes", _U8, (blocks, heads, page, half), dev)
    _need(vs, "v_scales", _U8, (blocks, heads, page, half // 16), dev)
    return KvCacheArgs(kc.data_ptr(), ks.data_ptr(), vc.data_ptr(), vs.data_ptr(), blocks, heads,
                       page, 2 * half)


def _vector(t, name, n, dev, dtypes=_I32):
    _need(t, name, dtypes, (n,), dev)
    return t.data_ptr()


def rfq_block_assign(ctx_lens, new_lens, block_tables, free_blocks, free_count, page, tokens,
                     stream=None):
    """Blocks, slots and positions of one step's tokens -> (slots [tokens],
    positions [tokens], seq_lens [B], query_starts [B + 1], counts [3]), all int32;
    block_tables [B][width] is updated.  counts: free blocks left, new tokens,
    refused requests.  seq_lens is 0 for a refused request, which keeps its tokens: the next
    step's ctx_lens is torch.maximum(ctx_lens, seq_lens).  The five may be parts of one
    allocation."""
    if stream is None:
        r = _native("block_assign", ctx_lens, new_lens, block_tables, free_blocks, free_count,
                    page, tokens)
        if r is not None:
            return r
    _need(ctx_lens, "ctx_lens", _I32)
    if ctx_lens.dim() != 1:
        raise ValueError("ctx_lens must be 1-D [B]")
    dev, B = ctx_lens.get_device(), ctx_lens.shape[0]
    _need(new_lens, "new_lens", _I32, (B,), dev)
    _need(block_tables, "block_tables", _I32, None, dev)
    _need(free_blocks, "free_blocks", _I32, None, dev)
    if block_tables.dim() != 2 or block_tables.shape[0] != B or free_blocks.dim() != 1:
        raise ValueError("block_tables must be [B][width] and free_blocks 1-D")
    _need(free_count, "free_count", _I32, (1,), dev)
    tokens = int(tokens)
    if tokens < 0:
        raise ValueError("tokens must not be negative")

    def new(n):
        return _empty(n, torch.int32, ctx_lens.device, stream)
    slots, positions, seq_lens, starts, counts = new(tokens), new(tokens), new(B), new(B + 1), new(3)
    st = load().rfq_block_assign(
        _ptr(ctx_lens), _ptr(new_lens), B, _ptr(block_tables), block_tables.shape[1],
        _ptr(free_blocks), free_blocks.shape[0], _ptr(free_count), int(page), tokens, _ptr(slots),
        _ptr(positions), _ptr(seq_lens), _ptr(starts), _ptr(counts), _stream(stream, dev))
    _check("rfq_block_assign", st)
    return slots, positions, seq_lens, starts, counts


def rfq_block_release(lens, ended, block_tables, free_blocks, free_count, page, stream=None):
    """Gives the blocks of the requests with ended != 0 (uint8 [B]) back to the list
    free_blocks (updated) -> its new count [1]."""
    if stream is None:
        r = _native("block_release", lens, ended, block_tables, free_blocks, free_count, page)
        if r is not None:
            return r
    _need(lens, "lens", _I32)
    if lens.dim() != 1:
        raise ValueError("lens must be 1-D [B]")
    dev, B = lens.get_device(), lens.shape[0]
    _need(ended, "ended", _U8, (B,), dev)
    _need(block_tables, "block_tables", _I32, None, dev)
    _need(free_blocks, "free_blocks", _I32, None, dev)
    if block_tables.dim() != 2 or block_tables.shape[0] != B or free_blocks.dim() != 1:
        raise ValueError("block_tables must be [B][width] and free_blocks 1-D")
    _need(free_count, "free_count", _I32, (1,), dev)
    count = _empty(1, torch.int32, lens.device, stream)
    st = load().rfq_block_release(
        _ptr(lens), _ptr(ended), B, _ptr(block_tables), block_tables.shape[1], _ptr(free_blocks),
        free_blocks.shape[0], _ptr(free_count), int(page), _ptr(count), _stream(stream, dev))
    _check("rfq_block_release", st)
    return count


class _Rope(torch.autograd.Function):
    """A rotation whose gradient is the rotation by the opposite angles."""

    @staticmethod
    def forward(ctx, x, positions, cos_sin, func, axes, interleaved):
        y = _rope_call(func, x, positions, cos_sin, axes, interleaved, None, None)
        ctx.save_for_backward(positions, cos_sin)
        ctx.rest = func, axes, interleaved
        return y

    @staticmethod
    def backward(ctx, dy):
        func, axes, interleaved = ctx.rest
        back = rfq_rope_backward if func == "rfq_rope" else rfq_rope
        strides = (dy.stride(0) * dy.element_size(), dy.stride(1) * dy.element_size())
        if dy.stride(2) != 1 or any(n % 16 for n in (dy.data_ptr(), *strides)):
            dy = dy.clone(memory_format=torch.contiguous_format)
        return back(dy, *ctx.saved_tensors, axes, interleaved), None, None, None, None, None


def _rope_call(func, x, positions, cos_sin, axes, interleaved, out, stream):
    if torch.is_grad_enabled() and isinstance(x, torch.Tensor) and (
            x.requires_grad or getattr(out, "requires_grad", False)):
        if out is not None:
            raise ValueError("out takes no gradient: x and out must not require one")
        args = (x, positions, cos_sin, func, axes, interleaved)
        if stream is None:
            return _Rope.apply(*args)
        # (Autograd runs the gradient on the stream that is current here.)
        with torch.cuda.stream(_torch_stream(stream, x.device)):
            y = _Rope.apply(*args)
        y.record_stream(torch.cuda.current_stream(x.device))
        return y
    if stream is None:
        r = _native(func[4:], x, positions, cos_sin, axes, interleaved, out)
        if r is not None:
            return r if out is None else _written(out)
    _need_heads(x, "x", _FLOAT)
    dev = x.get_device()
    T, H, D = x.shape
    spec = _rope(positions, cos_sin, axes, interleaved, T, dev)
    given = out
    if out is None:
        out = _empty((T, H, D), x.dtype, x.device, stream)
    else:
        _need_heads(out, "out", (x.dtype,), x.shape, dev)
    st = getattr(load(), func)(ctypes.byref(_heads(x)), _dtype_code(x), T, H, D,
                               ctypes.byref(spec), ctypes.byref(_heads(out)),
                               _stream(stream, dev))
    _check(func, st)
    return out if given is None else _written(out)


def rfq_rope(x, positions, cos_sin, axes=None, interleaved=False, out=None, stream=None):
    """x [T][H][D] (bf16 or fp32) with its first 2 * cos_sin.shape[1] channels
    rotated: pair j of token t by cos_sin[positions[axes[j]][t]][j].  positions
    int32 [axes][T] or [T]; axes: bytes or a sequence, one entry per pair (None:
    axis 0).  out may be x.  Differentiable in x (not in cos_sin), without out."""
    return _rope_call("rfq_rope", x, positions, cos_sin, axes, interleaved, out, stream)


def rfq_rope_backward(dy, positions, cos_sin, axes=None, interleaved=False, out=None,
                      stream=None):
    """The gradient of rfq_rope with respect to x, from that of its result.
    Differentiable in dy, without out."""
    return _rope_call("rfq_rope_backward", dy, positions, cos_sin, axes, interleaved, out, stream)


def rfq_kv_append(k, v, slots, cache, q=None, positions=None, cos_sin=None, axes=None,
                  interleaved=False, q_out=None, stream=None):
    """Quantizes k (rotated where positions and cos_sin are given) and v [T][heads][D]
    into the cache's slots [T]; negative slots are skipped.  With q [T][Hq][D]
    returns q rotated (q_out, or a new tensor), else None."""
    if stream is None:
        r = _native("kv_append", k, v, slots, *cache, q, positions, cos_sin, axes, interleaved,
                    q_out)
        if r is not None:
            return r[0] if q_out is None else _written(q_out)
    _need_heads(k, "k", _FLOAT)
    dev = k.get_device()
    T, heads, D = k.shape
    args = _need_cache(cache, dev)
    if heads != args.heads or D != args.D:
        raise ValueError("k has %d heads of %d channels, the cache %d of %d"
                         % (heads, D, args.heads, args.D))
    _need_heads(v, "v", (k.dtype,), k.shape, dev)
    _vector(slots, "slots", T, dev)
    if (positions is None) != (cos_sin is None):
        raise ValueError("positions and cos_sin must both be given or both be None")
    spec = None
    if positions is not None:
        spec = ctypes.byref(_rope(positions, cos_sin, axes, interleaved, T, dev))
    qa = qo = None
    Hq, given = 0, q_out
    if q is not None:
        if spec is None:
            raise ValueError("q is rotated: positions and cos_sin must be given")
        _need_heads(q, "q", (k.dtype,), None, dev)
        Hq = q.shape[1]
        if q.shape[0] != T or q.shape[2] != D:
            raise ValueError("q must be [%d][Hq][%d], not %s" % (T, D, tuple(q.shape)))
        if q_out is None:
            q_out = _empty((T, Hq, D), q.dtype, q.device, stream)
        else:
            _need_heads(q_out, "q_out", (q.dtype,), q.shape, dev)
        qa, qo = ctypes.byref(_heads(q)), ctypes.byref(_heads(q_out))
    elif q_out is not None:
        raise ValueError("q_out is given without q")
    st = load().rfq_kv_append(ctypes.byref(_heads(k)), ctypes.byref(_heads(v)), _dtype_code(k), T,
                              _ptr(slots), ctypes.byref(args), qa, Hq, spec, qo,
                              _stream(stream, dev))
    _check("rfq_kv_append", st)
    return q_out if given is None else _written(q_out)


def rfq_kv_gather(cache, slots, out_dtype=torch.bfloat16, stream=None):
    """The cached values of slots [n] -> (k, v), each [n][heads][D] (exact in bf16 and
    in fp32); zeros for a slot outside the cache."""
    if stream is None:
        r = _native("kv_gather", slots, *cache, _OUT_CODE.get(out_dtype, 2))
        if r is not None:
            return r
    _need(slots, "slots", _I32)
    if slots.dim() != 1:
        raise ValueError("slots must be 1-D [n]")
    if out_dtype not in _FLOAT:
        raise TypeError("out_dtype must be torch.float32 or torch.bfloat16")
    dev, n = slots.get_device(), slots.shape[0]
    args = _need_cache(cache, dev)
    k, v = (_empty((n, args.heads, args.D), out_dtype, slots.device, stream) for _ in range(2))
    st = load().rfq_kv_gather(ctypes.byref(args), _ptr(slots), n, _ptr(k), _ptr(v),
                              RFQ_BF16 if out_dtype == torch.bfloat16 else RFQ_F32,
                              _stream(stream, dev))
    _check("rfq_kv_gather", st)
    return k, v


def rfq_kv_attention_workspace_bytes(T, Hq, heads, D, B, max_query, max_seq):
    """Workspace of rfq_kv_attention for these sizes (0: nothing is split)."""
    return int(load().rfq_kv_attention_workspace_bytes(int(T), int(Hq), int(heads), int(D),
                                                       int(B), int(max_query), int(max_seq)))


def rfq_kv_attention(q, cache, block_tables, seq_lens, query_starts, max_query, max_seq,
                     scale=None, causal=True, window=0, return_lse=False, out=None,
                     workspace=None, stream=None):
    """Attention of the queries q [T][Hq][D] (bf16) of B requests over their cached
    tokens -> out [T][Hq][D] (bf16), with return_lse also the rows' log-sum-exp
    [T][Hq] (fp32).  Request b has the rows query_starts[b] .. query_starts[b + 1] - 1
    of q, its last seq_lens[b] tokens' queries.  max_query and max_seq (upper bounds of
    a request's queries and tokens) divide the work.  scale: 1 / sqrt(D) if None.
    workspace: a contiguous uint8 tensor of rfq_kv_attention_workspace_bytes, or None:
    one from torch's allocator."""
    if stream is None and isinstance(q, torch.Tensor) and q.dim() == 3 and q.shape[2] > 0:
        r = _native("kv_attention", q, *cache, block_tables, seq_lens, query_starts, max_query,
                    max_seq, float(q.shape[2] ** -0.5 if scale is None else scale), causal, window,
                    return_lse, out, workspace)
        if r is not None:
            if out is not None:
                _written(out)
            return r if return_lse else r[0]
    _need_heads(q, "q", _BF16)
    dev = q.get_device()
    T, Hq, D = q.shape
    args = _need_cache(cache, dev)
    if D != args.D:
        raise ValueError("q has %d channels a head, the cache %d" % (D, args.D))
    _need(block_tables, "block_tables", _I32, None, dev)
    if block_tables.dim() != 2:
        raise ValueError("block_tables must be 2-D [B][width]")
    B, width = block_tables.shape
    _vector(seq_lens, "seq_lens", B, dev)
    _vector(query_starts, "query_starts", B + 1, dev)
    given = out
    if out is None:
        out = _empty((T, Hq, D), q.dtype, q.device, stream)
    else:
        _need_heads(out, "out", _BF16, q.shape, dev)
    lse = _empty((T, Hq), torch.float32, q.device, stream) if return_lse else None
    if workspace is None:
        nbytes = load().rfq_kv_attention_workspace_bytes(T, Hq, args.heads, D, B, int(max_query),
                                                         int(max_seq))
        if nbytes > 0:
            workspace = _empty(nbytes, torch.uint8, q.device, stream, returned=False)
    else:
        _need(workspace, "workspace", _U8, None, dev)
        nbytes = workspace.numel()
    st = load().rfq_kv_attention(
        ctypes.byref(_heads(q)), T, Hq, ctypes.byref(args), _ptr(block_tables), width,
        _ptr(seq_lens), _ptr(query_starts), B, int(max_query), int(max_seq),
        D ** -0.5 if scale is None else float(scale), bool(causal), int(window),
        ctypes.byref(_heads(out)), _ptr(lse), _ptr(workspace), nbytes, _stream(stream, dev))
    _check("rfq_kv_attention", st)
    if given is not None:
        _written(out)
    return (out, lse) if return_lse else out
