"""Checks of linear attention with a decay and of the bias of distances that need no device: refusals of the C ABI and of the Python calls,
packed arguments, buckets."""
import ctypes as C
import math

import pytest
import torch
from torch.autograd import forward_ad

import paper_1911_00472_b200 as P
from paper_1911_00472_b200 import binding as B
from paper_1911_00472_b200 import mixing as M

E = B.PCR_E_ARG
FAR = 1 << 40                                    # made-up addresses lie far from one another


class Rows(C.Structure):
    _fields_ = [("at", C.c_void_p), ("stride", C.c_int64 * 3)]


class DecayArgs(C.Structure):
    _fields_ = [(n, Rows) for n in ("q", "k", "v", "out", "dq", "dk", "dv")] + [
        (n, C.c_void_p) for n in ("log_decay", "starts", "state", "state_after", "dstate_after", "dstate")] + [
        (n, C.c_int64) for n in ("batch", "tokens", "sequences")] + [(n, C.c_int32) for n in ("q_heads", "k_heads", "k_dim", "v_dim", "dtype", "flags")]


class StepArgs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "k", "v", "out")] + [(n, C.c_int64 * 2) for n in ("q_stride", "k_stride", "v_stride", "out_stride")] + [
        (n, C.c_void_p) for n in ("state", "slots", "log_decay")] + [(n, C.c_int64) for n in ("rows", "n_slots")] + [
        (n, C.c_int32) for n in ("q_heads", "k_heads", "k_dim", "v_dim", "dtype", "rsvd")]


class BiasArgs(C.Structure):
    _fields_ = [("table", C.c_void_p), ("bucket_of", C.c_void_p), ("q_positions", C.c_void_p), ("q_stride", C.c_int64 * 3), ("k_positions", C.c_void_p),
                ("k_stride", C.c_int64 * 3), ("q_ids", C.c_void_p), ("q_id_stride", C.c_int64 * 2), ("k_ids", C.c_void_p), ("k_id_stride", C.c_int64 * 2),
                ("bias", C.c_void_p), ("bias_stride", C.c_int64 * 3), ("batch", C.c_int64), ("q_tokens", C.c_int64), ("k_tokens", C.c_int64),
                ("heads", C.c_int32), ("axes", C.c_int32), ("buckets", C.c_int32), ("reach", C.c_int32), ("dtype", C.c_int32), ("table_dtype", C.c_int32)]


def decay_args():
    """Arguments that would pass: two batches of 100 tokens, 4 and 2 heads of 64 and 32 (their addresses are never followed)."""
    a = DecayArgs()
    for i, (n, heads, dim) in enumerate((("q", 4, 64), ("k", 2, 64), ("v", 2, 32), ("out", 4, 32), ("dq", 4, 64), ("dk", 2, 64), ("dv", 2, 32))):
        r = getattr(a, n)
        r.at = FAR + i * (1 << 30)
        r.stride[0], r.stride[1], r.stride[2] = 100 * heads * dim, heads * dim, dim
    a.log_decay = FAR + 9 * (1 << 30)
    a.batch, a.tokens, a.sequences, a.q_heads, a.k_heads, a.k_dim, a.v_dim, a.dtype = 2, 100, 2, 4, 2, 64, 32, B.PCR_BF16
    return a


def put(a, path, value):
    *way, last = path.split(".")
    for w in way:
        a = getattr(a, w)
    if last.isdigit():
        a[int(last)] = value
    else:
        setattr(a, last, value)


def set_in(a, path, value):
    if path.rsplit(".", 1)[-1].isdigit():
        head, i = path.rsplit(".", 1)
        b = a
        for w in head.split("."):
            b = getattr(b, w)
        b[int(i)] = value
    else:
        put(a, path, value)


def decay(a, back, scratch=FAR + 12 * (1 << 30)):
    raw = bytes(a)
    return (B.lib().pcr_decay_attention_backward if back else B.lib().pcr_decay_attention)(raw, scratch, None)


def test_layouts_of_packed_arguments():
    assert C.sizeof(DecayArgs) == M._DECAY_ARGS.size and C.sizeof(StepArgs) == M._STEP_ARGS.size and C.sizeof(BiasArgs) == M._BIAS_ARGS.size


WRONG = [("q_heads", 0), ("q_heads", 3), ("q_heads", 65536), ("k_heads", 0), ("k_heads", 8), ("k_dim", 0), ("k_dim", 257), ("v_dim", 0), ("v_dim", 300), ("dtype", 3), ("dtype", -1),
         ("flags", 2), ("batch", -1), ("tokens", -1), ("tokens", 1 << 31), ("batch", 1 << 31), ("sequences", 3), ("sequences", -1), ("sequences", 1 << 24), ("log_decay", 0), ("log_decay", FAR + 2),
         ("q.at", 0), ("k.at", 0), ("v.at", 0), ("out.at", 0), ("q.at", FAR + 1), ("starts", FAR + 10 * (1 << 30)), ("starts", FAR + 2), ("state", FAR + 10 * (1 << 30) + 1)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("field,value", WRONG)
def test_decay_refusals(field, value, back):
    a = decay_args()
    put(a, field, value)
    assert decay(a, back) == E
    assert B.lib().pcr_decay_scratch_bytes(bytes(a), back) == 0


@pytest.mark.parametrize("field,value,back", [("out.stride.1", 0, False), ("out.stride.2", 8, False), ("dq.stride.1", 64, True), ("dk.stride.2", 1, True), ("dv.stride.0", 0, True),
                                              ("dq.at", 0, True), ("dk.at", FAR + 1, True), ("state_after", FAR + 3, False), ("dstate", FAR + 3, True)])
def test_decay_outputs_that_overlap_themselves_or_are_not_there(field, value, back):
    a = decay_args()
    set_in(a, field, value)
    assert decay(a, back) == E


def test_decay_outputs_that_share_memory():
    for name, back in (("out", False), ("state_after", False), ("dq", True), ("dk", True), ("dv", True), ("dstate", True)):
        for other in ("q", "k", "v", "log_decay", "state", "starts") + (("out", "dstate_after") if back else ()):
            a = decay_args()
            a.state, a.dstate_after = FAR + 10 * (1 << 30), FAR + 11 * (1 << 30)
            if other == "starts":
                a.batch, a.sequences, a.starts = 1, 2, FAR + 13 * (1 << 30)
            at = getattr(a, other)
            at = at.at if isinstance(at, Rows) else at
            at += 8 if other in ("log_decay", "starts") else 64
            if name in ("state_after", "dstate"):
                setattr(a, name, at)
            else:
                getattr(a, name).at = at
            assert decay(a, back) == E, (name, other)
    a = decay_args()
    a.dk.at = a.dq.at + 128                       # two outputs
    assert decay(a, True) == E
    a = decay_args()
    a.tokens, a.batch, a.sequences = 100000, 1, 1  # long enough for several segments: scratch memory is needed, aligned and apart
    for r in ("q", "k", "v", "out"):
        getattr(a, r).at += 0
    assert B.lib().pcr_decay_scratch_bytes(bytes(a), 0) > 0
    assert decay(a, False, None) == E and decay(a, False, FAR + 12 * (1 << 30) + 4) == E and decay(a, False, a.q.at) == E and decay(a, False, a.out.at + 64) == E


def test_decay_of_nothing():
    a = decay_args()
    a.batch = a.sequences = 0
    a.log_decay = 0
    assert decay(a, False, None) == B.PCR_OK and decay(a, True, None) == B.PCR_OK and B.lib().pcr_decay_scratch_bytes(bytes(a), 0) == 0
    assert B.lib().pcr_decay_attention(None, None, None) == E and B.lib().pcr_decay_step(None, None) == E


def step_args():
    a = StepArgs()
    a.q, a.k, a.v, a.out, a.state, a.slots, a.log_decay = (FAR + i * (1 << 32) for i in range(7))
    for s, w in ((a.q_stride, 4 * 64), (a.k_stride, 2 * 64), (a.v_stride, 2 * 32), (a.out_stride, 4 * 32)):
        s[0], s[1] = w, 64 if w in (256, 128) and s is not a.out_stride else 32
    a.rows, a.n_slots, a.q_heads, a.k_heads, a.k_dim, a.v_dim, a.dtype = 5, 9, 4, 2, 64, 32, B.PCR_F16
    return a


@pytest.mark.parametrize("field,value", [("q_heads", 5), ("k_heads", 0), ("k_dim", 0), ("v_dim", 257), ("dtype", 9), ("rows", -1), ("rows", 1 << 24), ("n_slots", -1), ("n_slots", 1 << 31), ("q", 0), ("k", 0),
                                         ("v", 0), ("out", 0), ("state", 0), ("log_decay", 0), ("q", FAR + 1), ("state", FAR + 2), ("slots", FAR + 2), ("out_stride.0", 0), ("out_stride.1", 16),
                                         ("out", FAR + 4 * (1 << 32) + 64), ("out", FAR + 64), ("state", FAR + (1 << 32) + 64), ("out", FAR + 5 * (1 << 32) + 8)])
def test_step_refusals(field, value):
    a = step_args()
    set_in(a, field, value)
    assert B.lib().pcr_decay_step(bytes(a), None) == E


def test_step_without_slots_needs_a_memory_for_every_row():
    a = step_args()
    a.slots, a.n_slots = 0, 4
    assert B.lib().pcr_decay_step(bytes(a), None) == E
    a.rows = 0
    assert B.lib().pcr_decay_step(bytes(a), None) == B.PCR_OK


def bias_args():
    a = BiasArgs()
    a.table, a.bucket_of, a.q_positions, a.k_positions, a.bias = (FAR + i * (1 << 32) for i in range(5))
    a.q_stride[0], a.q_stride[1], a.q_stride[2] = 2 * 30, 30, 1
    a.k_stride[0], a.k_stride[1], a.k_stride[2] = 2 * 50, 50, 1
    a.bias_stride[0], a.bias_stride[1], a.bias_stride[2] = 3 * 30 * 50, 30 * 50, 50
    a.batch, a.q_tokens, a.k_tokens, a.heads, a.axes, a.buckets, a.reach, a.dtype, a.table_dtype = 2, 30, 50, 3, 2, 16, 8, B.PCR_BF16, B.PCR_BF16
    return a


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("field,value", [("heads", 0), ("heads", 4097), ("axes", 0), ("axes", 5), ("buckets", 0), ("buckets", 513), ("reach", -1), ("reach", (1 << 20) + 1), ("dtype", 3), ("table_dtype", 5),
                                         ("batch", -1), ("batch", 65536), ("q_tokens", -1), ("k_tokens", (1 << 30) + 1), ("table", 0), ("table", FAR + 1), ("bucket_of", 0), ("bucket_of", FAR + 2),
                                         ("q_positions", 0), ("k_positions", 0), ("k_positions", FAR + 1), ("bias", 0), ("bias", FAR + 1), ("q_ids", FAR + 7 * (1 << 32)), ("k_ids", FAR + 7 * (1 << 32)),
                                         ("bias", FAR + 64), ("table", FAR + 4 * (1 << 32) + 64)])
def test_bias_refusals(field, value, back):
    a = bias_args()
    put(a, field, value)
    raw = bytes(a)
    assert (B.lib().pcr_relative_bias_backward(raw, FAR + 8 * (1 << 32), None) if back else B.lib().pcr_relative_bias(raw, None)) == E


def test_bias_outputs_and_scratch():
    L = B.lib()
    a = bias_args()
    a.table_dtype = B.PCR_F16                     # a table of the other 16-bit type
    assert L.pcr_relative_bias(bytes(a), None) == E
    for i, v in ((0, 0), (1, 8), (2, 49)):
        a = bias_args()
        a.bias_stride[i] = v
        assert L.pcr_relative_bias(bytes(a), None) == E
    for at in ("bucket_of", "q_positions", "k_positions"):
        a = bias_args()
        a.bias = getattr(a, at) + 8
        assert L.pcr_relative_bias(bytes(a), None) == E
    a = bias_args()
    assert L.pcr_relative_bias_scratch_bytes(bytes(a)) > 0
    for scratch in (None, FAR + 8 * (1 << 32) + 4, a.bias, a.table, a.q_positions):
        assert L.pcr_relative_bias_backward(bytes(a), scratch, None) == E
    a.q_tokens = 0
    assert L.pcr_relative_bias(bytes(a), None) == B.PCR_OK
    assert L.pcr_relative_bias(None, None) == E and L.pcr_relative_bias_backward(None, None, None) == E


@pytest.mark.parametrize("batch,q_tokens,k_tokens,heads", [(32768, 1, 1 << 27, 4), (65535, 1, 1 << 30, 4), (65535, 1, 1 << 30, 4096), (32768, 1, 1 << 25, 64), (40000, 3, 1 << 26, 4)])
def test_bias_gradients_of_many_batches_that_share_all(batch, q_tokens, k_tokens, heads):
    """Strides of 0 stand for any number of batches: the scratch memory holds a sum for every one of the slabs, however many there are."""
    a = bias_args()
    a.batch, a.q_tokens, a.k_tokens, a.heads = batch, q_tokens, k_tokens, heads
    a.table = 1 << 60
    for s in (a.q_stride, a.k_stride):
        s[0], s[1], s[2] = 0, 0, 0
    a.bias_stride[0] = a.bias_stride[1] = a.bias_stride[2] = 0
    one = a.axes * a.buckets * heads * 4
    got = B.lib().pcr_relative_bias_scratch_bytes(bytes(a))
    assert got % one == 0 and 1 <= got // one < 1 << 31


def test_bias_of_more_pairs_than_are_counted():
    a = bias_args()
    a.batch, a.q_tokens, a.k_tokens = 16, 1 << 30, 1 << 30        # 2^64 of them: 0 in 64 bits
    raw = bytes(a)
    L = B.lib()
    assert L.pcr_relative_bias(raw, None) == E and L.pcr_relative_bias_scratch_bytes(raw) == 0 and L.pcr_relative_bias_backward(raw, FAR + 8 * (1 << 32), None) == E


# ---- the Python calls ------------------------------------------------------------------------------------------------------------


def heads(**change):
    a = dict(q=torch.zeros(10, 4, 16), k=torch.zeros(10, 2, 16), v=torch.zeros(10, 2, 8), log_decay=torch.zeros(4))
    a.update(change)
    return a


@pytest.mark.parametrize("change,match", [
    (dict(q=torch.zeros(10, 4, 16).double()), "float16"), (dict(k=torch.zeros(10, 2, 16).half()), "alike"), (dict(k=torch.zeros(9, 2, 16)), "queries and keys"),
    (dict(v=torch.zeros(10, 1, 8)), "queries and keys"), (dict(k=torch.zeros(10, 2, 8)), "queries and keys"), (dict(k=torch.zeros(10, 3, 16), v=torch.zeros(10, 3, 8)), "multiple"),
    (dict(log_decay=torch.zeros(2)), "log_decay"), (dict(log_decay=torch.zeros(4).double()), "log_decay"), (dict(v=torch.zeros(10, 2, 300)), "256"),
    (dict(starts=torch.zeros(3)), "starts"), (dict(starts=torch.zeros(0, dtype=torch.int32)), "starts"), (dict(state=torch.zeros(1, 4, 16, 4)), "state"),
    (dict(state=torch.zeros(1, 4, 16, 8).half()), "state"), (dict(state=torch.zeros(1, 4, 8, 16).transpose(2, 3)), "state"),
    (dict(q=torch.zeros(10, 4, 16, requires_grad=True)), "autograd"), (dict(v=torch.zeros(10, 2, 8, requires_grad=True)), "autograd"), (dict(log_decay=torch.zeros(4, requires_grad=True)), "autograd"),
    (dict(state=torch.zeros(1, 4, 16, 8, requires_grad=True)), "autograd"), ({}, "CUDA device")])
def test_attention_refusals(change, match):
    with pytest.raises(ValueError, match=match):
        P.decay_attention(**heads(**change))
    a = heads(**change)
    with pytest.raises(ValueError, match=match):
        P.decay_attention_backward(torch.zeros(*a["q"].shape[:-1], a["v"].shape[-1], dtype=a["q"].dtype), **a)


def test_more_attention_refusals():
    with pytest.raises(ValueError, match="no batch"):
        P.decay_attention(torch.zeros(2, 10, 4, 16), torch.zeros(2, 10, 2, 16), torch.zeros(2, 10, 2, 8), torch.zeros(4), starts=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="grad must"):
        P.decay_attention_backward(torch.zeros(10, 4, 9), **heads())
    with pytest.raises(ValueError, match="grad_final"):
        P.decay_attention_backward(torch.zeros(10, 4, 8), **heads(), grad_final=torch.zeros(2, 4, 16, 8))
    with forward_ad.dual_level(), pytest.raises(ValueError, match="autograd"):
        P.decay_attention(**heads(k=forward_ad.make_dual(torch.zeros(10, 2, 16), torch.ones(10, 2, 16))))
    a = heads()
    for state in (torch.zeros(9, 4, 16, 8), torch.zeros(10, 4, 8, 16), torch.zeros(10, 4, 16, 8).half()):
        with pytest.raises(ValueError, match="state"):
            P.decay_step(a["q"], a["k"], a["v"], a["log_decay"], state)
    with pytest.raises(ValueError, match="slots"):
        P.decay_step(a["q"], a["k"], a["v"], a["log_decay"], torch.zeros(3, 4, 16, 8), slots=torch.zeros(10, dtype=torch.int64))


def bias(**change):
    a = dict(table=torch.zeros(2, 16, 4), buckets=torch.zeros(9, dtype=torch.int32), q_positions=torch.zeros(2, 5, dtype=torch.int32), k_positions=torch.zeros(2, 7, dtype=torch.int32))
    a.update(change)
    return a


@pytest.mark.parametrize("change,match", [
    (dict(table=torch.zeros(3, 16, 4)), "table"), (dict(table=torch.zeros(2, 16, 4).double()), "table"), (dict(table=torch.zeros(2, 4, 16).transpose(1, 2)), "table"),
    (dict(buckets=torch.zeros(8, dtype=torch.int32)), "buckets"), (dict(buckets=torch.zeros(9)), "buckets"), (dict(q_positions=torch.zeros(2, 5)), "positions"),
    (dict(k_positions=torch.zeros(1, 7, dtype=torch.int32)), "positions"), (dict(q_positions=torch.zeros(5, dtype=torch.int32)), "positions"), (dict(q_ids=torch.zeros(5, dtype=torch.int32)), "go together"),
    (dict(q_ids=torch.zeros(4, dtype=torch.int32), k_ids=torch.zeros(7, dtype=torch.int32)), "ids"), (dict(table=torch.zeros(2, 16, 4).half(), dtype=torch.float32), "dtype"),
    (dict(table=torch.zeros(2, 16, 4, requires_grad=True)), "autograd"), ({}, "CUDA device")])
def test_bias_call_refusals(change, match):
    with pytest.raises(ValueError, match=match):
        P.relative_bias(**bias(**change))


def test_ids_of_the_columns_are_those_of_the_rows():
    """Where there are as many tokens, also of positions of their own (the next thing that is looked at is the device)."""
    a = bias(k_positions=torch.ones(2, 5, dtype=torch.int32), q_ids=torch.zeros(5, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA device"):
        P.relative_bias(**a)
    del a["table"]
    with pytest.raises(ValueError, match="CUDA device"):
        P.relative_bias_backward(torch.zeros(4, 5, 5), 16, **a)


def test_bias_gradient_call_refusals():
    a = bias()
    del a["table"]
    for grad, kw, match in ((torch.zeros(4, 5, 6), {}, "grad"), (torch.zeros(4, 5, 7).double(), {}, "grad"), (torch.zeros(5, 7), {}, "grad"), (torch.zeros(4, 5, 7), dict(dtype=torch.float64), "dtype"),
                            (torch.zeros(4, 5, 7, requires_grad=True), {}, "autograd"), (torch.zeros(4, 5, 7), {}, "CUDA device")):
        with pytest.raises(ValueError, match=match):
            P.relative_bias_backward(grad, 16, **a, **kw)
    with pytest.raises(ValueError, match="buckets"):
        P.relative_bias_backward(torch.zeros(4, 5, 7), 0, **a)
    b = torch.zeros(2, 3, 5, dtype=torch.int32)    # positions of three batches, gradients of two
    with pytest.raises(ValueError, match="grad"):
        P.relative_bias_backward(torch.zeros(2, 4, 5, 5), 16, a["buckets"], b)


def test_buckets():
    got = P.relative_buckets(32, 128, device="cpu").tolist()
    assert len(got) == 257 and got[128] == 0 and got[128 - 7:128] == [7, 6, 5, 4, 3, 2, 1] and got[129:136] == [17, 18, 19, 20, 21, 22, 23] and got[0] == 15 and got[256] == 31
    for d in range(-128, 129):                     # the definition, distance by distance
        a, n = abs(d), 16 if d > 0 else 0
        want = n + (a if a < 8 else min(15, 8 + int(math.log(a / 8) / math.log(128 / 8) * 8 + 1e-9)))
        assert got[128 + d] == want
    one = P.relative_buckets(8, 20, one_sided=True, device="cpu").tolist()
    assert one[20:] == [0] * 21 and one[16:20] == [4, 3, 2, 1] and one[0] == 7 and sorted(set(one)) == list(range(8))
    assert P.relative_buckets(4, 1, device="cpu").tolist() == [1, 0, 3] and len(P.relative_buckets(2, 1, one_sided=True, device="cpu")) == 3
    for bad in ((7, 10), (2, 10), (32, 7), (0, 0)):
        with pytest.raises(ValueError):
            P.relative_buckets(*bad, device="cpu")
