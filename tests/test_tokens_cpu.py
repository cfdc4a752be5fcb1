"""Checks of the token operators that need no device: refusals of the C ABI, packed arguments, plans and axes."""
import ctypes as C
import math
import struct

import numpy as np
import pytest
import torch

import paper_1911_00472_b200 as P
from paper_1911_00472_b200 import binding as B
from paper_1911_00472_b200 import tokens as T

E = B.PCR_E_ARG


class Heads(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("dy", C.c_void_p), ("weight", C.c_void_p), ("dweight", C.c_void_p),
                ("x_stride", C.c_int64 * 3), ("y_stride", C.c_int64 * 3), ("dy_stride", C.c_int64 * 3), ("heads", C.c_int32), ("rsvd", C.c_int32)]


class TurnArgs(C.Structure):
    _fields_ = [("q", Heads), ("k", Heads), ("positions", C.c_void_p), ("position_stride", C.c_int64 * 3), ("inv_freq", C.c_void_p), ("axes", C.c_void_p),
                ("batch", C.c_int64), ("tokens", C.c_int64), ("n_axes", C.c_int32), ("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("interleaved", C.c_int32),
                ("inverse", C.c_int32), ("dtype", C.c_int32), ("freq_dtype", C.c_int32), ("weight_dtype", C.c_int32), ("eps", C.c_float), ("rsvd", C.c_int32)]


def good():
    """Arguments that would pass (the addresses are never followed: every call below is refused, or has nothing to do)."""
    a = TurnArgs()
    for h in (a.q, a.k):
        h.x = h.y = h.dy = h.weight = h.dweight = 4096
        h.heads = 2
        for s in (h.x_stride, h.y_stride, h.dy_stride):
            s[0], s[1], s[2] = 5 * 128, 128, 64
    a.positions = a.inv_freq = a.axes = 4096
    a.batch, a.tokens, a.n_axes, a.head_dim, a.rot_dim = 3, 5, 3, 64, 64
    a.dtype, a.freq_dtype, a.weight_dtype, a.eps = B.PCR_BF16, B.PCR_F64, B.PCR_F32, 1e-6
    return a


def calls(a):
    L = B.lib()
    raw = bytes(a)
    return L.pcr_rotate(raw, None), L.pcr_norm_rotate(raw, None), L.pcr_norm_rotate_backward(raw, 4096, None), L.pcr_norm_rotate_scratch_bytes(raw)


def test_packed_arguments_have_the_layout_of_the_struct():
    assert T._TURN_ARGS.size == C.sizeof(TurnArgs) == 344
    a = good()
    fields = []
    for h in (a.q, a.k):
        fields += [h.x, h.y, h.dy, h.weight, h.dweight, *h.x_stride, *h.y_stride, *h.dy_stride, h.heads, 0]
    fields += [a.positions, *a.position_stride, a.inv_freq, a.axes, a.batch, a.tokens, a.n_axes, a.head_dim, a.rot_dim, 0, 0, a.dtype, a.freq_dtype,
               a.weight_dtype, a.eps, 0]
    assert T._TURN_ARGS.pack(*fields) == bytes(a)


@pytest.mark.parametrize("name,value", [("head_dim", 0), ("head_dim", 513), ("head_dim", 62), ("rot_dim", 63), ("rot_dim", -2), ("rot_dim", 66), ("n_axes", 0),
                                        ("n_axes", 5), ("dtype", 3), ("dtype", -1), ("freq_dtype", 0), ("batch", -1), ("tokens", -1), ("batch", 1 << 30),
                                        ("tokens", 1 << 40), ("batch", 1 << 62), ("interleaved", 2), ("inverse", 2), ("positions", None), ("positions", 4097),
                                        ("inv_freq", None), ("inv_freq", 4100), ("axes", None), ("axes", 4098)])
def test_refused_by_every_call(name, value):
    a = good()
    setattr(a, name, value)
    assert calls(a) == (E, E, E, 0)


@pytest.mark.parametrize("name,value", [("eps", -1.0), ("eps", math.inf), ("eps", math.nan), ("weight_dtype", B.PCR_F16), ("weight_dtype", 7), ("inverse", 1)])
def test_refused_by_the_backward_norms(name, value):
    a = good()
    setattr(a, name, value)
    L, raw = B.lib(), bytes(a)
    assert (L.pcr_norm_rotate(raw, None), L.pcr_norm_rotate_backward(raw, 4096, None), L.pcr_norm_rotate_scratch_bytes(raw)) == (E, E, 0)


@pytest.mark.parametrize("part", ["q", "k"])
@pytest.mark.parametrize("name,value", [("x", None), ("y", None), ("x", 4097), ("y", 4099), ("heads", -1), ("heads", 65536)])
def test_refused_operands(part, name, value):
    a = good()
    setattr(getattr(a, part), name, value)
    assert calls(a) == (E, E, E, 0)


@pytest.mark.parametrize("name,value", [("dy", None), ("dy", 4097), ("weight", None), ("dweight", 4098), ("weight", 4098)])
def test_refused_by_the_backward_pass(name, value):
    a = good()
    setattr(a.q, name, value)
    L, raw = B.lib(), bytes(a)
    assert (L.pcr_norm_rotate_backward(raw, 4096, None), L.pcr_norm_rotate_scratch_bytes(raw)) == (E, 0)


@pytest.mark.parametrize("strides", [(640, 128, 0), (640, 128, 63), (640, 64, 64), (640, 127, 64), (639, 128, 64), (0, 128, 64), (64, 128, 64), (640, -127, 64)])
def test_outputs_that_overlap_themselves(strides):
    a = good()
    a.k.y_stride[:] = strides
    assert calls(a) == (E, E, E, 0)


def test_scratch_has_to_be_given_where_weights_have_gradients():
    a = good()
    assert B.lib().pcr_norm_rotate_scratch_bytes(bytes(a)) > 0
    assert B.lib().pcr_norm_rotate_backward(bytes(a), None, None) == E
    assert B.lib().pcr_norm_rotate_backward(bytes(a), 4098, None) == E


def test_nothing_to_do_needs_no_device():
    L = B.lib()
    for part in ("batch", "tokens", "heads"):
        a = good()
        if part == "heads":
            a.q.heads = a.k.heads = 0
        else:
            setattr(a, part, 0)
        raw = bytes(a)
        assert (L.pcr_rotate(raw, None), L.pcr_norm_rotate(raw, None), L.pcr_norm_rotate_scratch_bytes(raw)) == (0, 0, 0)
    assert L.pcr_rotate(None, None) == E and L.pcr_norm_rotate(None, None) == E and L.pcr_norm_rotate_backward(None, None, None) == E


def test_patch_tokens_refuses():
    m, s = struct.pack("3f", 0.5, 0.5, 0.5), struct.pack("3f", 0.2, 0.2, 0.2)
    ok = [4096, 1000, 4096, 2, 4096, 10, 14, 2, m, s, B.PCR_BF16, 4096, None]
    call = B.lib().pcr_patch_tokens
    for at, bad in [(0, None), (0, 4097), (2, None), (2, 4104), (3, -1), (4, None), (4, 4100), (5, -1), (5, 1 << 31), (6, 0), (6, 33), (7, 0), (7, 65), (8, None),
                    (9, None), (9, struct.pack("3f", 0.2, 0.0, 0.2)), (9, struct.pack("3f", 0.2, math.nan, 0.2)), (8, struct.pack("3f", math.inf, 0, 0)),
                    (10, 3), (11, None), (11, 4097)]:
        args = list(ok)
        args[at] = bad
        assert call(*args) == E, (at, bad)
    args = list(ok)
    args[5] = 0
    assert call(*args) == 0


def test_token_positions_refuses():
    ok = [4096, 3, 100, 2, 1, 1, 0, 4096, 100, 4096, 4096, None]
    call = B.lib().pcr_token_positions
    for at, bad in [(0, None), (0, 4104), (1, -1), (2, -1), (2, 1 << 31), (3, -1), (4, 0), (4, 65), (5, -1), (5, (1 << 20) + 1), (6, 4), (7, None), (7, 4098), (8, 99),
                    (9, None), (9, 4097), (10, 4100)]:
        args = list(ok)
        args[at] = bad
        assert call(*args) == E, (at, bad)
    need = B.lib().pcr_token_positions_scratch_bytes
    assert need(-1) == 0 and need(3) == 0 and need(20000) >= 12 * 20001
    args = list(ok)
    args[1], args[10] = 20000, None               # so many segments need scratch memory
    assert call(*args) == E


def test_operands_on_the_host_are_refused():
    q = torch.zeros(4, 2, 8)
    f, a = P.rotary_axes(8, device="cpu")
    with pytest.raises(ValueError):
        P.rotate(q, None, torch.zeros(1, 4, dtype=torch.int32), f, a)
    with pytest.raises(ValueError):
        P.token_positions(torch.zeros(1, 4, dtype=torch.int32), 1, 1)
    with pytest.raises(ValueError):
        P.patch_tokens(torch.zeros(8, dtype=torch.uint8), torch.zeros(1, 10, dtype=torch.int64), torch.zeros(1, 2, dtype=torch.int32), 14, (0,) * 3, (1,) * 3)
    with pytest.raises(ValueError):
        P.rotate(q.requires_grad_(), None, torch.zeros(1, 4, dtype=torch.int32), f, a)


@pytest.mark.parametrize("mean,std", [((0.5,) * 2, (1,) * 3), ((0.5,) * 3, (1,) * 4)])
def test_means_of_other_than_three_channels_are_refused(mean, std):
    with pytest.raises(ValueError, match="three"):
        P.patch_tokens(torch.zeros(8, dtype=torch.uint8), torch.zeros(1, 10, dtype=torch.int64), torch.zeros(1, 2, dtype=torch.int32), 14, mean, std)


def test_axes():
    f, a = P.rotary_axes(16, base=100.0, sections=(2, 3, 3), device="cpu")
    assert a.tolist() == [0, 0, 1, 1, 1, 2, 2, 2] and f.dtype == torch.float64 and a.dtype == torch.int32
    assert np.allclose(f.numpy(), 100.0 ** (-np.arange(8) / 8), rtol=1e-15)
    assert P.rotary_axes(16, sections=(2, 3, 3), interleaved_axes=True, device="cpu")[1].tolist() == [0, 1, 2, 0, 1, 2, 1, 2]
    f, a = P.rotary_axes(12, sections=(0, 3, 3), per_axis=True, device="cpu")
    assert a.tolist() == [1, 1, 1, 2, 2, 2] and np.allclose(f.numpy(), np.tile(10000.0 ** (-np.arange(3) / 3), 2), rtol=1e-15)
    assert P.rotary_axes(0, device="cpu")[0].numel() == 0
    for bad in (dict(rot=7), dict(rot=8, sections=(2, 1)), dict(rot=8, sections=(5, -1)), dict(rot=10, sections=(1,) * 5)):
        with pytest.raises(ValueError):
            P.rotary_axes(device="cpu", **bad)


class Info:
    def __init__(self, out_offset, width, height):
        self.out_offset, self.width, self.height = out_offset, width, height


def test_plan():
    info = [Info(0, 30, 57), Info(5376, 1, 1), Info(5504, 28, 28)]
    plan = P.patch_plan(info, 14, merge=2, device="cpu")
    assert plan.grids.tolist() == [[4, 2], [2, 2], [2, 2]]
    assert plan.images.tolist()[0] == [0, 30, 57, 0, 0, 30, 57, 4, 2, 0]
    assert plan.index.shape == (16, 2) and plan.index[:, 1].tolist() == list(range(8)) + list(range(4)) * 2
    assert plan.segments().tolist() == [[1, 4, 2, 0], [1, 2, 2, 1], [1, 2, 2, 2]]
    assert plan.segments(merged=True).tolist() == [[1, 2, 1, 0], [1, 1, 1, 1], [1, 1, 1, 2]]
    plan = P.patch_plan(info[:1], 8, crops=np.array([[3, 7, 20, 40, 1]]), grids=np.array([[5, 3]]), device="cpu")
    assert plan.images.tolist() == [[0, 30, 57, 3, 7, 20, 40, 5, 3, 1]]
    assert P.patch_plan([], 14, device="cpu").index.shape == (0, 2)
    for bad in (dict(patch=0), dict(patch=33), dict(patch=14, merge=0), dict(patch=14, merge=2, grids=np.array([[3, 2]] * 3)), dict(patch=14, grids=np.array([[0, 2]] * 3)),
                dict(patch=14, crops=np.zeros((3, 5))), dict(patch=14, crops=np.array([[0, 0, 2, 1, 0]] * 3)), dict(patch=14, grids=np.array([[1, 1]])),
                dict(patch=32, grids=np.array([[1 << 16, 1]] * 3))):
        with pytest.raises(ValueError):
            P.patch_plan(info, device="cpu", **bad)
