"""What a sequence model does with its tokens' heads and positions: linear attention whose memory fades at a rate of each
head's own, and a learned bias of the distance between two tokens.

torch is used for memory and streams only; all arithmetic happens behind the C ABI (include/pcr.h: pcr_decay_attention,
pcr_decay_attention_backward, pcr_decay_step, pcr_relative_bias, pcr_relative_bias_backward).  Nothing is kept between calls and
nothing waits, so every call may be captured into a graph; relative_buckets apart, which makes a map on the host and copies it, once for a
model.  Gradients are calls of their own: operands that autograd follows are
refused, not silently cut off.

Work goes to `stream` (default: torch's current stream of the operands' device); what a call allocates belongs to it.
"""
from __future__ import annotations

import math
import struct

import torch

from . import binding as B
from .tokens import _CODES, _current_device, _forward_mode, _has_tangent, _not_followed, _on, _raw_stream, _written

_DECAY_ARGS = struct.Struct("<28Q6Q3q6i")           # pcr_decay_args
_STEP_ARGS = struct.Struct("<4Q8q3Q2q6i")           # pcr_decay_step_args
_BIAS_ARGS = struct.Struct("<3Q3qQ3qQ2qQ2qQ3q3q6i")  # pcr_bias_args
_NO_ROWS = (0, 0, 0, 0)


def _operands(tensors, stream):
    """One device, none that autograd follows (it does not see these calls), signs resolved (once the call is on its own device and stream):
    the tensors to read from."""
    device, followed, negated = None, False, False
    for t in tensors:
        if t is None:
            continue
        if device is None:
            device = t.device
        elif t.device != device:
            raise ValueError("all operands have to be on one device")
        followed = followed or t.requires_grad
        negated = negated or t.is_neg()
    if (followed and torch.is_grad_enabled()) or (_forward_mode() and _has_tangent(tensors)):
        raise ValueError("autograd does not see this call: detach the operands and call the backward pass yourself")
    if device.type != "cuda":
        raise ValueError("operands have to be on a CUDA device")
    if negated and stream is None and _current_device() == device.index:
        tensors = [None if t is None else t.resolve_neg() for t in tensors]
    return device, tensors


def _side_by_side(t):
    return t if t is None or t.stride(-1) == 1 or t.shape[-1] <= 1 else t.contiguous()


def _output(out, shape, dtype, device, what, contiguous=False):
    if out.shape != tuple(shape) or out.dtype != dtype:
        raise ValueError(f"{what} must have shape {tuple(shape)} and dtype {dtype}")
    if out.device != device:
        raise ValueError("all operands have to be on one device")
    if contiguous and not out.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if out.shape[-1] > 1 and out.stride(-1) != 1:
        raise ValueError(f"the elements of a head of {what} must stand side by side")
    _not_followed(out)


def _rows(t):
    """pcr_rows of a (tokens, heads, size) or (batch, tokens, heads, size) tensor."""
    s = t.stride()
    return (t.data_ptr(), 0, s[0], s[1]) if len(s) == 3 else (t.data_ptr(), *s[:3])


def _at(t):
    return 0 if t is None else t.data_ptr()


# ---- linear attention with a decay for each head ----------------------------------------------------------------------------


def _decay_shapes(q, k, v, log_decay, starts, rank):
    """(batch, tokens, sequences, heads of queries, of keys, sizes of keys and values); `rank`: dimensions that come before the heads."""
    if q.dtype not in _CODES or q.dtype != k.dtype or q.dtype != v.dtype:
        raise ValueError("queries, keys and values must be float16, bfloat16 or float32, all alike")
    if q.dim() not in rank or k.dim() != q.dim() or v.dim() != q.dim() or k.shape[:-2] != q.shape[:-2] or v.shape[:-1] != k.shape[:-1] or k.shape[-1] != q.shape[-1]:
        raise ValueError("queries and keys must be (*tokens, heads, size), values (*tokens, heads of the keys, size)")
    hq, kd = q.shape[-2:]
    hk, vd = v.shape[-2:]
    if hk < 1 or hq < 1 or hq % hk:
        raise ValueError("the heads of the queries must be a multiple of those of the keys")
    if not 1 <= kd <= 256 or not 1 <= vd <= 256:
        raise ValueError("heads must have 1 to 256 elements")
    if log_decay.shape != (hq,) or log_decay.dtype != torch.float32 or not log_decay.is_contiguous():
        raise ValueError("log_decay must be a contiguous float32 vector, an element for each head of the queries")
    if starts is not None:
        if q.dim() != 3:
            raise ValueError("packed sequences have no batch: starts belongs to (tokens, heads, size)")
        if starts.dim() != 1 or starts.dtype != torch.int32 or starts.shape[0] < 1 or not starts.is_contiguous():
            raise ValueError("starts must be a contiguous int32 vector of one element more than there are sequences")
    batch, tokens = (1, q.shape[0]) if q.dim() == 3 else q.shape[:2]
    return batch, tokens, batch if starts is None else starts.shape[0] - 1, hq, hk, kd, vd


def _memory(t, shape, what):
    if t is not None and (t.shape != shape or t.dtype != torch.float32 or not t.is_contiguous()):
        raise ValueError(f"{what} must be contiguous float32 of shape {shape}")


def _decay_call(name, backward, rows, scalars, states, sizes, dtype, flags, device, like):
    args = _DECAY_ARGS.pack(*(x for t in rows for x in (_NO_ROWS if t is None else _rows(t))), *map(_at, scalars), *map(_at, states), *sizes, _CODES[dtype], flags)
    L = B.lib()
    scratch = like.new_empty(-(-L.pcr_decay_scratch_bytes(args, backward) // 4), dtype=torch.float32)
    B._chk(getattr(L, name)(args, scratch.data_ptr(), _raw_stream(device.index)), name)


def decay_attention(q, k, v, log_decay, *, starts=None, state=None, final=False, out=None, stream=None):
    """Linear attention whose memory fades: (outputs, memories behind the last tokens or None).

        S_t = exp(log_decay) S_(t-1) + k_t v_t^T        out_t = S_t^T q_t

    q, k, v    (tokens, heads, size) or (batch, tokens, heads, size) of any strides (slices of one projection's output, or what
               rotate and norm_rotate give); only where a head's elements do not stand side by side are they copied
               first.  Consecutive heads of the queries share one of the keys and values, whose size may be another
    log_decay  (heads of the queries,) float32, at most 0
    starts     (n + 1,) int32 on the device: (tokens, heads, size) are n packed sequences, tokens starts[i] .. starts[i + 1] - 1 each;
               without it every batch is a sequence
    state      (sequences, heads, key size, value size) float32: memories to begin with
    final      whether the memories behind the last tokens are wanted, or where they go
    out        where the outputs go: rows of no sequence stay as they are there; without it they are 0

    Memories are in single precision.  16-bit operands go through the tensor cores where their layout allows it, and some products
    on the way are rounded to their type then (include/pcr.h says which): the same values in another layout may differ by that.
    """
    batch, tokens, n, hq, hk, kd, vd = _decay_shapes(q, k, v, log_decay, starts, (3, 4))
    memories = (n, hq, kd, vd)
    _memory(state, memories, "state")
    device, (q, k, v, log_decay, starts, state) = _operands((q, k, v, log_decay, starts, state), stream)
    if out is not None:
        _output(out, (*q.shape[:-1], vd), q.dtype, device, "out")
    given = torch.is_tensor(final)
    if given:
        _output(final, memories, torch.float32, device, "final", True)
    if stream is not None or _current_device() != device.index:
        with _on(device, stream):
            return decay_attention(q, k, v, log_decay, starts=starts, state=state, final=final, out=out)
    q, k, v = map(_side_by_side, (q, k, v))
    y = q.new_empty((*q.shape[:-1], vd)) if out is None else out
    after = final if given else q.new_empty(memories, dtype=torch.float32) if final else None
    _decay_call("pcr_decay_attention", 0, (q, k, v, y, None, None, None), (log_decay, starts), (state, after, None, None),
                (batch, tokens, n, hq, hk, kd, vd), q.dtype, B.PCR_DECAY_ZERO_TAIL if out is None else 0, device, q)
    written = [t for t in (out, final if given else None) if t is not None]
    if written:
        _written(written)
    return y, after


def decay_attention_backward(grad, q, k, v, log_decay, *, starts=None, state=None, grad_final=None, grad_state=False, out=None, stream=None):
    """Gradients of decay_attention from that of its outputs and from its inputs: (q, k, v, state or None).

    grad_final   gradient of the memories behind the last tokens, None: 0
    grad_state   whether the gradient of the memories to begin with is wanted (None otherwise); state None: of zeros
    out          where the gradients of q, k and v go: rows of no sequence stay as they are there; without it they are 0
    """
    batch, tokens, n, hq, hk, kd, vd = _decay_shapes(q, k, v, log_decay, starts, (3, 4))
    memories = (n, hq, kd, vd)
    _memory(state, memories, "state")
    _memory(grad_final, memories, "grad_final")
    if grad.shape != (*q.shape[:-1], vd) or grad.dtype != q.dtype:
        raise ValueError("grad must have the shape and the dtype of the outputs")
    device, (grad, q, k, v, log_decay, starts, state, grad_final) = _operands((grad, q, k, v, log_decay, starts, state, grad_final), stream)
    if out is not None:
        for o, x, what in zip(out, (q, k, v), ("out[0]", "out[1]", "out[2]"), strict=True):
            _output(o, x.shape, x.dtype, device, what)
    if stream is not None or _current_device() != device.index:
        with _on(device, stream):
            return decay_attention_backward(grad, q, k, v, log_decay, starts=starts, state=state, grad_final=grad_final, grad_state=grad_state, out=out)
    grad, q, k, v = map(_side_by_side, (grad, q, k, v))
    dq, dk, dv = (x.new_empty(x.shape) for x in (q, k, v)) if out is None else out
    before = q.new_empty(memories, dtype=torch.float32) if grad_state else None
    _decay_call("pcr_decay_attention_backward", 1, (q, k, v, grad, dq, dk, dv), (log_decay, starts), (state, None, grad_final, before),
                (batch, tokens, n, hq, hk, kd, vd), q.dtype, B.PCR_DECAY_ZERO_TAIL if out is None else 0, device, q)
    if out is not None:
        _written(tuple(out))
    return dq, dk, dv, before


def decay_step(q, k, v, log_decay, state, *, slots=None, out=None, stream=None):
    """decay_attention for one new token of each request: its memory is brought up to date where it lies; returns the outputs.

    q, k, v    (requests, heads, size), see decay_attention
    state      (memories, heads, key size, value size) contiguous float32, written
    slots      (requests,) int32 on the device: the request's memory; one that is none (-1) stands for a row of no request, whose
               output is 0; rows of one memory are taken one after the other.  None: request i has memory i
    """
    rows, _, _, hq, hk, kd, vd = _decay_shapes(q, k, v, log_decay, None, (3,))
    rows = q.shape[0]
    if state.dim() != 4 or state.shape[1:] != (hq, kd, vd) or state.dtype != torch.float32 or not state.is_contiguous():
        raise ValueError(f"state must be contiguous float32 of shape (memories, {hq}, {kd}, {vd})")
    if slots is None:
        if state.shape[0] < rows:
            raise ValueError("state must have a memory for every request")
    elif slots.shape != (rows,) or slots.dtype != torch.int32 or not slots.is_contiguous():
        raise ValueError("slots must be a contiguous int32 vector, an element for each request")
    device, (q, k, v, log_decay, slots) = _operands((q, k, v, log_decay, slots), stream)
    if state.device != device:
        raise ValueError("all operands have to be on one device")
    _not_followed(state)
    if out is not None:
        _output(out, (rows, hq, vd), q.dtype, device, "out")
    if stream is not None or _current_device() != device.index:
        with _on(device, stream):
            return decay_step(q, k, v, log_decay, state, slots=slots, out=out)
    q, k, v = map(_side_by_side, (q, k, v))
    y = q.new_empty((rows, hq, vd)) if out is None else out
    args = _STEP_ARGS.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), y.data_ptr(), *q.stride()[:2], *k.stride()[:2], *v.stride()[:2], *y.stride()[:2],
                           state.data_ptr(), _at(slots), log_decay.data_ptr(), rows, state.shape[0], hq, hk, kd, vd, _CODES[q.dtype], 0)
    B._chk(B.lib().pcr_decay_step(args, _raw_stream(device.index)), "pcr_decay_step")
    _written((state,) if out is None else (state, out))
    return y


# ---- a bias of distances --------------------------------------------------------------------------------------------------------


def relative_buckets(buckets, reach, *, one_sided=False, device="cuda:0"):
    """Bucket (2 * reach + 1,) int32 of every distance -reach .. reach: single distances up to half of a side's buckets, then
    distances that grow by a factor, up to `reach`, from which on all share the last one.  Made on the host: not for a capture.

    one_sided   keys that come later than their query share bucket 0, all buckets are for earlier ones; otherwise the first half
                is for earlier keys and the query itself, the second for later ones
    """
    side = buckets if one_sided else buckets // 2
    single = side // 2
    if single < 1 or reach < single or (not one_sided and buckets % 2):
        raise ValueError("buckets must be even and at least 4 (2 where they are one-sided), reach at least a quarter of them (half)")
    got = []
    for d in range(-reach, reach + 1):
        a = abs(d)
        n = a if a < single else side - 1 if reach == single else min(side - 1, single + int(math.log(a / single) / math.log(reach / single) * (side - single) + 1e-9))
        got.append((0 if one_sided else n + side) if d > 0 else n)
    return torch.tensor(got, dtype=torch.int32, device=device)


def _bias_shapes(buckets, q_positions, k_positions, q_ids, k_ids):
    """(axes, batch or None, tokens of the rows, of the columns)"""
    if buckets.dim() != 1 or buckets.shape[0] % 2 == 0 or buckets.dtype != torch.int32 or not buckets.is_contiguous():
        raise ValueError("buckets must be a contiguous int32 vector of 2 * reach + 1 elements")
    if q_positions.dtype != torch.int32 or k_positions.dtype != torch.int32 or q_positions.dim() not in (2, 3) or k_positions.shape[:-1] != q_positions.shape[:-1]:
        raise ValueError("positions must be int32, (axes, tokens) or (axes, batch, tokens), of rows and columns alike")
    if (q_ids is None) != (k_ids is None):
        raise ValueError("q_ids and k_ids go together")
    for ids, positions in ((q_ids, q_positions), (k_ids, k_positions)):
        if ids is not None and (ids.dtype != torch.int32 or ids.shape != positions.shape[1:]):
            raise ValueError("ids must be int32 and have the shape of an axis of the positions")
    return q_positions.shape[0], q_positions.shape[1] if q_positions.dim() == 3 else None, q_positions.shape[-1], k_positions.shape[-1]


def _bias_pack(table, buckets, q_positions, k_positions, q_ids, k_ids, rows, batch, nq, nk, heads, axes, n_buckets):
    def places(t):
        s = t.stride()
        return (t.data_ptr(), *(s if len(s) == 3 else (s[0], 0, s[1])))

    def ids(t):
        return (0, 0, 0) if t is None else (t.data_ptr(), *(t.stride() if t.dim() == 2 else (0, t.stride(0))))

    return _BIAS_ARGS.pack(table.data_ptr(), buckets.data_ptr(), *places(q_positions), *places(k_positions), *ids(q_ids), *ids(k_ids),
                           rows.data_ptr(), *(rows.stride()[:3] if rows.dim() == 4 else (0, *rows.stride()[:2])), batch, nq, nk, heads, axes, n_buckets,
                           buckets.shape[0] // 2, _CODES[rows.dtype], _CODES[table.dtype])


def relative_bias(table, buckets, q_positions, k_positions=None, *, q_ids=None, k_ids=None, dtype=None, out=None, stream=None):
    """A learned bias for every head and pair of tokens, by the buckets of their distance on each axis:

        bias[..., h, i, j] = sum over axes a of table[a, buckets[reach + clamp(k_positions[a, ..., j] - q_positions[a, ..., i])], h]

    table        (axes, buckets, heads), contiguous
    buckets      (2 * reach + 1,) int32: the bucket of every distance -reach .. reach (relative_buckets makes them); those beyond are
                 taken as the ends; a bucket that the table does not have counts as 0
    positions    (axes, tokens) or (axes, batch, tokens) int32, any strides; k_positions None: the same as q_positions
    ids          int32, of an axis's shape: pairs whose ids differ are minus infinity (packed sequences); k_ids None: as q_ids, for as
                 many tokens
    dtype        of the bias: the table's (default), or any where the table is float32
    Returns (heads, rows, columns) or (batch, heads, rows, columns); out: where they go, a row's elements side by side
    """
    if k_positions is None:
        k_positions = q_positions
    if k_ids is None and k_positions.shape == q_positions.shape:
        k_ids = q_ids
    axes, batch, nq, nk = _bias_shapes(buckets, q_positions, k_positions, q_ids, k_ids)
    dtype = dtype or table.dtype
    if table.dim() != 3 or table.shape[0] != axes or table.dtype not in _CODES or not table.is_contiguous():
        raise ValueError("table must be contiguous (axes, buckets, heads) of float16, bfloat16 or float32")
    if dtype not in _CODES or (table.dtype != dtype and table.dtype != torch.float32):
        raise ValueError("dtype must be float16, bfloat16 or float32, the table's or any where that is float32")
    heads = table.shape[2]
    shape = (heads, nq, nk) if batch is None else (batch, heads, nq, nk)
    device, (table, buckets, q_positions, k_positions, q_ids, k_ids) = _operands((table, buckets, q_positions, k_positions, q_ids, k_ids), stream)
    if out is not None:
        _output(out, shape, dtype, device, "out")
    if stream is not None or _current_device() != device.index:
        with _on(device, stream):
            return relative_bias(table, buckets, q_positions, k_positions, q_ids=q_ids, k_ids=k_ids, dtype=dtype, out=out)
    y = table.new_empty(shape, dtype=dtype) if out is None else out
    args = _bias_pack(table, buckets, q_positions, k_positions, q_ids, k_ids, y, 1 if batch is None else batch, nq, nk, heads, axes, table.shape[1])
    B._chk(B.lib().pcr_relative_bias(args, _raw_stream(device.index)), "pcr_relative_bias")
    if out is not None:
        _written(out)
    return y


def relative_bias_backward(grad, n_buckets, buckets, q_positions, k_positions=None, *, q_ids=None, k_ids=None, dtype=torch.float32, stream=None):
    """Gradient (axes, n_buckets, heads) of relative_bias's table, of `dtype`, from that of the bias (whatever masked places hold).

    grad   (heads, rows, columns) or (batch, heads, rows, columns) of any strides; only where a row's elements do not stand side by
           side is it copied first.  Positions and ids without a batch stand for all batches
    """
    if k_positions is None:
        k_positions = q_positions
    if k_ids is None and k_positions.shape == q_positions.shape:
        k_ids = q_ids
    axes, batch, nq, nk = _bias_shapes(buckets, q_positions, k_positions, q_ids, k_ids)
    if grad.dim() not in (3, 4) or grad.dtype not in _CODES or grad.shape[-2:] != (nq, nk) or (batch is not None and (grad.dim() == 3 or grad.shape[0] != batch)):
        raise ValueError("grad must be (heads, rows, columns) or (batch, heads, rows, columns) of the positions, float16, bfloat16 or float32")
    if dtype not in _CODES or n_buckets < 1:
        raise ValueError("dtype must be float16, bfloat16 or float32, and there must be buckets")
    heads = grad.shape[-3]
    device, (grad, buckets, q_positions, k_positions, q_ids, k_ids) = _operands((grad, buckets, q_positions, k_positions, q_ids, k_ids), stream)
    if stream is not None or _current_device() != device.index:
        with _on(device, stream):
            return relative_bias_backward(grad, n_buckets, buckets, q_positions, k_positions, q_ids=q_ids, k_ids=k_ids, dtype=dtype)
    grad = _side_by_side(grad)
    dtable = grad.new_empty((axes, n_buckets, heads), dtype=dtype)
    args = _bias_pack(dtable, buckets, q_positions, k_positions, q_ids, k_ids, grad, grad.shape[0] if grad.dim() == 4 else 1, nq, nk, heads, axes, n_buckets)
    L = B.lib()
    scratch = grad.new_empty(-(-L.pcr_relative_bias_scratch_bytes(args) // 4), dtype=torch.float32)
    B._chk(L.pcr_relative_bias_backward(args, scratch.data_ptr(), _raw_stream(device.index)), "pcr_relative_bias_backward")
    return dtable
