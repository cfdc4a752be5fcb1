"""From decoded pixels to a sequence model: patch tokens, positions on several axes, and the queries and keys they turn.

torch is used for memory and streams only; all arithmetic happens behind the C ABI (include/pcr.h: pcr_patch_tokens,
pcr_token_positions, pcr_rotate, pcr_norm_rotate, pcr_norm_rotate_backward).  Nothing is kept between calls and nothing
waits, so every call may be captured into a graph.  Gradients are calls of their own (rotate with inverse=True,
norm_rotate_backward): operands that autograd follows are refused, not silently cut off.

Work goes to `stream` (default: torch's current stream of the operands' device); what a call allocates belongs to it.
"""
from __future__ import annotations

import contextlib
import struct
from typing import NamedTuple

import numpy as np
import torch
from torch.autograd import forward_ad

from . import binding as B

_CODES = {torch.float16: B.PCR_F16, torch.float32: B.PCR_F32, torch.bfloat16: B.PCR_BF16}
_FREQ_CODES = {torch.float32: B.PCR_F32, torch.float64: B.PCR_F64}
_TURN_ARGS = struct.Struct("<5Q9q2i5Q9q2iQ3qQQqq8ifi")         # pcr_turn_args
_NO_HEADS, _NO_STRIDES = (0,) * 16, (0,) * 4


@contextlib.contextmanager
def _switched(device, stream):
    with torch.cuda.device(device):
        if stream is None:
            yield
        else:
            with torch.cuda.stream(stream):
                yield


_HERE = contextlib.nullcontext()
# the handle of a device's current stream, without the object around it: a third of what a small call costs
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)

# (the operands are on a device: nothing is left to set up)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on(device: torch.device, stream):
    """The context in which a call allocates and launches: the operands' device, and `stream` where one is given."""
    if device.type != "cuda":
        raise ValueError("operands have to be on a CUDA device")
    if stream is None and _current_device() == device.index:
        return _HERE
    if stream is not None and stream.device != device:
        raise ValueError("the stream belongs to another device than the operands")
    return _switched(device, stream)


def _has_tangent(tensors) -> bool:
    """Whether forward-mode differentiation follows one of them (asked where a level of it is entered: see _forward_mode)."""
    return any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


def _forward_mode() -> bool:
    return getattr(forward_ad, "_current_level", 0) >= 0


def _not_followed(out):
    """Outputs are written without autograd's knowledge: none may stand in its graph, or have its sign taken on reading."""
    if out.is_neg():
        raise ValueError("out must not be a negated view")
    if (out.requires_grad and torch.is_grad_enabled()) or (_forward_mode() and _has_tangent((out,))):
        raise ValueError("autograd does not see this call: out must be detached")


# tells autograd that a caller's tensors hold other values now: a graph that kept one of them says so when it needs it
_written = torch.autograd.graph.increment_version


def _same_device(device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError("all operands have to be on one device")


# ---- queries and keys ---------------------------------------------------------------------------------------------------


def _check(q, k, positions, inv_freq, axes, q_weight, k_weight, grads):
    """What the calls ask of their operands; returns (batch, tokens, size, heads of queries and of keys, positions' axes, pairs, type
    of the weights, whether an operand's sign is taken on reading).  One look at each property: small calls take as long as the
    host does."""
    shape, dtype, device = q.shape, q.dtype, q.get_device()
    k_heads = 0
    if len(shape) == 4:
        batch, tokens, q_heads, size = shape
    elif len(shape) == 3:
        batch, (tokens, q_heads, size) = 1, shape
    else:
        batch = tokens = q_heads = size = None
    if size is None or dtype not in _CODES:
        raise ValueError("queries must be (tokens, heads, size) or (batch, tokens, heads, size) of float16, bfloat16 or float32")
    if k is not None:
        other = k.shape
        if len(other) != len(shape) or other[-3] != tokens or other[-1] != size or other[0] != shape[0] or k.dtype != dtype:
            raise ValueError("k must have the tokens, head size and dtype of the queries")
        k_heads = other[-2]
    other = positions.shape
    if len(other) != len(shape) - 1 or other[-1] != tokens or other[1] != shape[0] or positions.dtype != torch.int32:
        raise ValueError("positions must be int32 with shape (axes, *tokens)")
    n_axes, other = other[0], inv_freq.shape
    if len(other) != 1 or inv_freq.dtype not in _FREQ_CODES or not inv_freq.is_contiguous():
        raise ValueError("inv_freq must be a contiguous float32 or float64 vector")
    if axes.shape != other or axes.dtype != torch.int32 or not axes.is_contiguous():
        raise ValueError("axes must be a contiguous int32 vector as long as inv_freq")
    near = device == positions.get_device() == inv_freq.get_device() == axes.get_device() and (k is None or k.get_device() == device)
    followed = q.requires_grad or inv_freq.requires_grad or (k is not None and k.requires_grad)
    negated = q.is_neg() or inv_freq.is_neg() or (k is not None and k.is_neg())
    weight = dtype
    if q_weight is not None or k_weight is not None:
        weight = (k_weight if q_weight is None else q_weight).dtype
        for w in (q_weight, k_weight):
            if w is not None:
                if w.shape != (size,) or w.dtype != weight or (weight != dtype and weight != torch.float32) or not w.is_contiguous():
                    raise ValueError("weights must be contiguous vectors of the head size, of the operands' type or float32, both alike")
                near = near and w.get_device() == device
                followed = followed or w.requires_grad
                negated = negated or w.is_neg()
        if k is None and k_weight is not None:
            raise ValueError("k_weight without keys")
    for g, x in zip(grads, (q, k)):
        if (g is None) != (x is None) or (x is not None and (g.shape != x.shape or g.dtype != dtype)):
            raise ValueError("gradients must have the shapes and the dtype of their operands")
        if g is not None:
            near = near and g.get_device() == device
            followed = followed or g.requires_grad
            negated = negated or g.is_neg()
    if not near:
        raise ValueError("all operands have to be on one device")
    if (followed and torch.is_grad_enabled()) or (_forward_mode() and _has_tangent((q, k, inv_freq, q_weight, k_weight, *grads))):
        raise ValueError("autograd does not see this call: detach the operands and call the backward pass yourself")
    return batch, tokens, size, q_heads, k_heads, n_axes, other[0], weight, negated


def _like(t):
    """An output of the operand's strides where its heads' elements stand side by side, a contiguous one otherwise."""
    return torch.empty_like(t) if t.stride(-1) == 1 else torch.empty_like(t, memory_format=torch.contiguous_format)


def _outputs(q, k, out):
    if out is None:
        return _like(q), None if k is None else _like(k)
    device = q.get_device()
    for o, x in zip(out, (q, k), strict=True):
        if (o is None) != (x is None):
            raise ValueError("out must have an output for each operand")
        if x is not None:
            if o.shape != x.shape or o.dtype != x.dtype:
                raise ValueError("out must have the shapes and the dtype of the operands")
            if o.shape[-1] > 1 and o.stride(-1) != 1:
                raise ValueError("the elements of a head of out must stand side by side")
            if o.get_device() != device:
                raise ValueError("all operands have to be on one device")
            _not_followed(o)
    return out


def _call(name, q, k, grads, q_weight, k_weight, positions, inv_freq, axes, interleaved, inverse, eps, out, stream):
    """Checks, allocates, packs a pcr_turn_args and makes the call `name`; returns its outputs (and the weights' gradients)."""
    batch, tokens, size, q_heads, k_heads, n_axes, pairs, weight, negated = _check(q, k, positions, inv_freq, axes, q_weight, k_weight, grads)
    device = q.get_device()
    if device < 0:
        raise ValueError("operands have to be on a CUDA device")
    if stream is not None or _current_device() != device:
        with _on(q.device, stream):
            return _call(name, q, k, grads, q_weight, k_weight, positions, inv_freq, axes, interleaved, inverse, eps, out, None)
    if negated:                                          # their memory holds the other sign
        q_, k_, wq_, wk_, freq_, *grads_ = (None if t is None else t.resolve_neg() for t in (q, k, q_weight, k_weight, inv_freq, *grads))
        return _call(name, q_, k_, tuple(grads_), wq_, wk_, positions, freq_, axes, interleaved, inverse, eps, out, None)
    y, z = _outputs(q, k, out)
    dwq = dwk = None
    if grads and q_weight is not None:
        dwq = torch.empty_like(q_weight)
    if grads and k_weight is not None:
        dwk = torch.empty_like(k_weight)
    parts, copies = [], []                               # (copies live until the call is made: others must not get their memory before)
    for x, o, g, w, dw, heads in ((q, y, grads[0] if grads else None, q_weight, dwq, q_heads), (k, z, grads[1] if grads else None, k_weight, dwk, k_heads)):
        if x is None:
            parts += _NO_HEADS
            continue
        xs = x.stride()
        if xs[-1] != 1 and size > 1:                     # the elements of a head do not stand side by side
            x = x.contiguous()
            xs = x.stride()
            copies.append(x)
        gs, g_at = _NO_STRIDES, 0
        if g is not None:
            gs = g.stride()
            if gs[-1] != 1 and size > 1:
                g = g.contiguous()
                gs = g.stride()
                copies.append(g)
            g_at = g.data_ptr()
        ys = o.stride()
        if len(xs) == 3:
            xs, ys, gs = (0, *xs), (0, *ys), (0, *gs)
        parts += (x.data_ptr(), o.data_ptr(), g_at, 0 if w is None else w.data_ptr(), 0 if dw is None else dw.data_ptr(), *xs[:3], *ys[:3], *gs[:3], heads, 0)
    ps = positions.stride()
    args = _TURN_ARGS.pack(*parts, positions.data_ptr(), *(ps if len(ps) == 3 else (ps[0], 0, ps[1])), inv_freq.data_ptr(), axes.data_ptr(), batch, tokens,
                           n_axes, size, 2 * pairs, bool(interleaved), bool(inverse), _CODES[q.dtype], _FREQ_CODES[inv_freq.dtype],
                           _CODES[weight], eps, 0)
    L = B.lib()
    if grads:
        scratch = inv_freq.new_empty(-(-L.pcr_norm_rotate_scratch_bytes(args) // inv_freq.element_size()))
        B._chk(L.pcr_norm_rotate_backward(args, scratch.data_ptr(), _raw_stream(device)), name)
    else:
        B._chk(getattr(L, name)(args, _raw_stream(device)), name)
    if out is not None:
        _written((y,) if z is None else (y, z))
    return (y, z, dwq, dwk) if grads else (y, z)


def rotate(q, k, positions, inv_freq, axes, *, interleaved=False, inverse=False, out=None, stream=None):
    """Queries and keys turned by the positions of their tokens.

    q, k      (tokens, heads, size) or (batch, tokens, heads, size) of any strides (slices of one projection's output);
              only where a head's elements do not stand side by side are they copied first; k may be None or have
              another number of heads
    positions (n_axes, *tokens) int32, any strides (expanded batches too)
    inv_freq, axes   frequency and axis of every pair of elements (rotary_axes makes them); the first 2 * len(inv_freq)
              elements of a head are turned, the others copied
    interleaved      pairs (2 i, 2 i + 1) in place of (i, i + len(inv_freq))
    inverse   by the negative angle: the gradient of the forward call
    out       (q, k) to write to: each its own operand, or memory that shares nothing with any operand or with the
              other output (anything else is refused)
    """
    return _call("pcr_rotate", q, k, (), None, None, positions, inv_freq, axes, interleaved, inverse, 0.0, out, stream)


def norm_rotate(q, k, q_weight, k_weight, positions, inv_freq, axes, *, eps=1e-6, interleaved=False, out=None, stream=None):
    """Queries and keys behind a root-mean-square norm of every head, then turned (see rotate), in one pass.

    q_weight, k_weight   (size,) of the operands' type or float32; None: ones
    """
    return _call("pcr_norm_rotate", q, k, (), q_weight, k_weight, positions, inv_freq, axes, interleaved, False, eps, out, stream)


def norm_rotate_backward(grad_q, grad_k, q, k, q_weight, k_weight, positions, inv_freq, axes, *, eps=1e-6, interleaved=False,
                         out=None, stream=None):
    """Gradients of norm_rotate from those of its outputs and from its inputs: (q, k, q_weight, k_weight).

    out   where the gradients of q and k go; grad_q or q itself allowed for the first, grad_k or k for the second (see rotate)
    """
    return _call("pcr_norm_rotate_backward", q, k, (grad_q, grad_k), q_weight, k_weight, positions, inv_freq, axes, interleaved, False, eps, out, stream)


def rotary_axes(rot, base=10000.0, sections=None, *, interleaved_axes=False, per_axis=False, device="cuda:0"):
    """(inv_freq, axes) of `rot` turned elements, rot / 2 pairs.

    sections          pairs of each axis (their sum is rot / 2); None: one axis
    interleaved_axes  the axes take turns, one that has no pairs left is passed over; otherwise the sections are runs
    per_axis          every axis has the whole range of frequencies over its own pairs (image encoders), otherwise
                      frequency i is base ** (-2 i / rot) whatever the axis
    """
    half = rot // 2
    sections = [half] if sections is None else list(sections)
    if rot % 2 or rot < 0 or sum(sections) != half or min(sections) < 0 or len(sections) > 4:
        raise ValueError("sections must be up to four counts of pairs that add up to rot / 2")
    if interleaved_axes:
        left, axes = list(sections), []
        while len(axes) < half:
            for a in range(len(left)):
                if left[a]:
                    left[a] -= 1
                    axes.append(a)
    else:
        axes = [a for a, n in enumerate(sections) for _ in range(n)]
    seen, freq = [0] * len(sections), []
    for i, a in enumerate(axes):
        freq.append(base ** (-seen[a] / sections[a]) if per_axis else base ** (-i / half))
        seen[a] += 1
    return torch.tensor(freq, dtype=torch.float64, device=device), torch.tensor(axes, dtype=torch.int32, device=device)


# ---- positions ------------------------------------------------------------------------------------------------------------


def token_positions(segments, n_tokens, n_sequences, *, merge=1, time_step=1, restart=False, out=None, stream=None):
    """Positions (3, n_tokens) of packed sequences and the position (n_sequences,) with which each goes on, both int32.

    segments    (n, 4) int32 on the device: time (or tokens), height, width, sequence; text has no height or width, the
                rows of a sequence stand together
    merge       grids are numbered in blocks of merge x merge, as patches are
    time_step   positions between two frames of a grid
    restart     every segment begins at 0 (an image encoder's positions)
    out         (3, at least n_tokens) int32 to write to: columns behind the last token stay as they are; without it they are 0
    """
    if segments.dtype != torch.int32 or segments.dim() != 2 or segments.shape[1] != 4 or not segments.is_contiguous():
        raise ValueError("segments must be a contiguous (n, 4) int32 tensor")
    if out is not None and (out.dtype != torch.int32 or out.dim() != 2 or out.shape[0] != 3 or out.shape[1] < n_tokens or out.stride(1) != 1):
        raise ValueError("out must be int32 of shape (3, n_tokens) with a row's elements side by side")
    _same_device(segments.device, out)
    given = out
    with _on(segments.device, stream):
        flags = B.PCR_POSITIONS_RESTART if restart else 0
        if out is None:
            flags |= B.PCR_POSITIONS_ZERO_TAIL
            out = segments.new_empty((3, n_tokens))
        after = segments.new_empty(n_sequences)
        L = B.lib()
        need = L.pcr_token_positions_scratch_bytes(segments.shape[0])
        scratch = segments.new_empty(-(-need // 4)) if need else after
        B._chk(L.pcr_token_positions(segments.data_ptr(), segments.shape[0], n_tokens, n_sequences, merge, time_step, flags, out.data_ptr(),
                                     out.stride(0), after.data_ptr(), scratch.data_ptr(), _raw_stream(segments.device.index)),
               "pcr_token_positions")
    if given is not None:
        _written(given)
    return out, after


# ---- patches --------------------------------------------------------------------------------------------------------------


def patch_tokens(rgb, images, index, patch, mean, std, *, merge=1, dtype=torch.bfloat16, out=None, stream=None):
    """Patch tokens (n_tokens, 3 * patch * patch) of the images of a decode's output.

    rgb      uint8 output of a decode
    images   (n, 10) int64 on the device, a row per image: first byte, width, height, rectangle x0, y0, w, h, patches down
             and across, flip
    index    (n_tokens, 2) int32 on the device: image and patch of every token; an entry that does not fit gives zeros
    merge    patches are numbered in blocks of merge x merge
    """
    if rgb.dtype != torch.uint8 or rgb.dim() != 1 or not rgb.is_contiguous():
        raise ValueError("rgb must be a contiguous uint8 vector")
    if images.dtype != torch.int64 or images.dim() != 2 or images.shape[1] != 10 or not images.is_contiguous():
        raise ValueError("images must be a contiguous (n, 10) int64 tensor")
    if index.dtype != torch.int32 or index.dim() != 2 or index.shape[1] != 2 or not index.is_contiguous():
        raise ValueError("index must be a contiguous (n, 2) int32 tensor")
    if dtype not in _CODES:
        raise ValueError("dtype must be torch.float16, torch.bfloat16 or torch.float32")
    if len(mean) != 3 or len(std) != 3:
        raise ValueError("mean and std must have three values")
    shape = (index.shape[0], 3 * patch * patch)
    if out is not None and (out.shape != shape or out.dtype != dtype or not out.is_contiguous()):
        raise ValueError("out must be contiguous, (n_tokens, 3 * patch * patch) of dtype")
    _same_device(rgb.device, images, index, out)
    if out is not None:
        _not_followed(out)
    given = out
    with _on(rgb.device, stream):
        if out is None:
            out = rgb.new_empty(shape, dtype=dtype)
        B._chk(B.lib().pcr_patch_tokens(rgb.data_ptr(), rgb.numel(), images.data_ptr(), images.shape[0], index.data_ptr(), shape[0], patch,
                                        merge, struct.pack("3f", *mean), struct.pack("3f", *std), _CODES[dtype], out.data_ptr(),
                                        _raw_stream(rgb.device.index)), "pcr_patch_tokens")
    if given is not None:
        _written(given)
    return out


class PatchPlan(NamedTuple):
    """What the images of a record become: tables on the device (see patch_tokens), and patches down and across on the host."""
    images: torch.Tensor
    index: torch.Tensor
    grids: np.ndarray
    patch: int
    merge: int

    def segments(self, merged: bool = False) -> torch.Tensor:
        """Segments of token_positions, an image a sequence: its patches, or (merged) its blocks of merge x merge."""
        m = self.merge if merged else 1
        n = len(self.grids)
        rows = np.stack([np.ones(n), self.grids[:, 0] // m, self.grids[:, 1] // m, np.arange(n)], 1).astype(np.int32)
        return torch.from_numpy(rows).to(self.index.device)


def patch_plan(info, patch, *, merge=1, crops=None, grids=None, device="cuda:0") -> PatchPlan:
    """Plan of the images of `info` (Decoder.info: out_offset, width, height).

    crops   (n, 5) x0, y0, w, h, flip as for Decoder.decode_tensor; None: the whole images
    grids   (n, 2) patches down and across; None: the rectangle's sides rounded to whole blocks, at least one
    """
    n = len(info)
    size = np.array([(i.out_offset, i.width, i.height) for i in info], dtype=np.int64).reshape(n, 3)
    if crops is None:
        crops = np.concatenate([np.zeros((n, 2), np.int64), size[:, 1:], np.zeros((n, 1), np.int64)], 1)
    crops = np.ascontiguousarray(crops, dtype=np.int64)
    if crops.shape != (n, 5):
        raise ValueError("crops must have shape (n_images, 5)")
    x0, y0, w, h, flip = crops.T
    if (crops[:, :2] < 0).any() or (crops[:, 2:4] < 1).any() or (x0 + w > size[:, 1]).any() or (y0 + h > size[:, 2]).any() or ((flip != 0) & (flip != 1)).any():
        raise ValueError("every rectangle must lie inside its image, flip 0 or 1")
    if not 1 <= patch <= 32 or not 1 <= merge <= 64:
        raise ValueError("patch must be 1..32, merge 1..64")
    unit = patch * merge
    if grids is None:
        grids = merge * np.maximum(1, (2 * crops[:, [3, 2]] + unit) // (2 * unit))
    grids = np.ascontiguousarray(grids, dtype=np.int64)
    if grids.shape != (n, 2) or (grids < 1).any() or (grids % merge).any() or (grids * patch > 1 << 20).any():
        raise ValueError("grids must have shape (n_images, 2), whole blocks of merge x merge patches, sides of 2^20 pixels at most")
    count = grids[:, 0] * grids[:, 1]
    if count.sum() >= 1 << 31:
        raise ValueError("too many tokens for one batch")
    image = np.repeat(np.arange(n), count)
    local = np.arange(len(image)) - np.repeat(np.cumsum(count) - count, count)
    table = np.concatenate([size, crops[:, :4], grids, crops[:, 4:]], 1)
    index = np.stack([image, local], 1).astype(np.int32)
    return PatchPlan(torch.from_numpy(table).to(device), torch.from_numpy(index).to(device), grids, patch, merge)
