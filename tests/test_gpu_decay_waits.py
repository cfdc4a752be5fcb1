"""Waits of the walks on the tensor cores that run out: nothing that was not worked out looks as if it had been.

The hook stops the copies of operands of each CTA behind some chunks, on the device, and lets waits end after a millisecond; nothing faults, and the
context goes on."""
import ctypes as C

import pytest
import torch

import paper_1911_00472_b200 as P
from paper_1911_00472_b200 import binding as B
from paper_1911_00472_b200 import mixing as M
from test_gpu_decay import DEV, make

pytestmark = pytest.mark.gpu
SEVEN = 7.0


def lost(back, rows, scalars, states, sizes, dtype, after):
    args = M._DECAY_ARGS.pack(*(x for t in rows for x in (M._NO_ROWS if t is None else M._rows(t))), *map(M._at, scalars), *map(M._at, states), *sizes, M._CODES[dtype], 0)
    L = B.lib()
    scratch = torch.full((max(1, -(-L.pcr_decay_scratch_bytes(args, back) // 4)),), SEVEN, device=DEV)       # what nobody writes is a number
    return L.pcr_selftest_decay_waits(args, back, scratch.data_ptr(), after, torch.cuda.current_stream().cuda_stream)


def whole_or_lost(got, want, what):
    """Rows of the last axis: as they should be, bit by bit, or all NaN; how many were lost."""
    none = got.isnan().all(-1)
    assert ((got == want).all(-1) | none).all(), what
    return int(none.sum())


# lengths, heads of queries, of keys, size: more segments than there are CTAs at a time, so that some have taken several; long ones in several
# segments; packed and batched
SHAPES = [([1000] * 4, 64, 64, 64, False), ([700, 300, 0, 129, 500, 1], 64, 32, 128, True), ([20000], 2, 1, 64, False), ([9000, 100, 5000], 1, 1, 128, True)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("after", [0, 1, 3, 10, 21])
@pytest.mark.parametrize("shape", SHAPES, ids=["batch", "packed", "long", "long_packed"])
def test_forward(shape, after, dtype):
    lengths, hq, hk, size, packed = shape
    q, k, v, _, starts, log_decay, first, _ = make(lengths, hq, hk, size, size, dtype, packed=packed, seed=21)
    want, memory = P.decay_attention(q, k, v, log_decay, starts=starts, state=first, final=True)
    out, last = torch.full_like(want, SEVEN), torch.full_like(memory, SEVEN)
    tokens = sum(lengths) if packed else lengths[0]
    sizes = (1 if packed else len(lengths), tokens, len(lengths), hq, hk, size, size)
    assert lost(0, (q, k, v, out, None, None, None), (log_decay, starts), (first, last, None, None), sizes, dtype, after) == B.PCR_OK
    torch.cuda.synchronize()
    n = whole_or_lost(out, want, "out") + whole_or_lost(last.flatten(-2), memory.flatten(-2), "memory")
    assert n > 0 or after > 0                                        # (further on, only where a CTA walks over more than that)
    again, _ = P.decay_attention(q, k, v, log_decay, starts=starts, state=first, final=True)
    assert torch.equal(again, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("after", [0, 2, 12])
@pytest.mark.parametrize("shape", SHAPES, ids=["batch", "packed", "long", "long_packed"])
def test_backward(shape, after, dtype):
    lengths, hq, hk, size, packed = shape
    q, k, v, g, starts, log_decay, first, dafter = make(lengths, hq, hk, size, size, dtype, packed=packed, seed=23)
    want = P.decay_attention_backward(g, q, k, v, log_decay, starts=starts, state=first, grad_final=dafter, grad_state=True)
    got = [torch.full_like(x, SEVEN) for x in want]
    tokens = sum(lengths) if packed else lengths[0]
    sizes = (1 if packed else len(lengths), tokens, len(lengths), hq, hk, size, size)
    assert lost(1, (q, k, v, g, *got[:3]), (log_decay, starts), (first, None, dafter, got[3]), sizes, dtype, after) == B.PCR_OK
    torch.cuda.synchronize()
    n = sum(whole_or_lost(x, y, i) for i, (x, y) in enumerate(zip(got[:3], want[:3]))) + whole_or_lost(got[3].flatten(-2), want[3].flatten(-2), "dstate")
    assert n > 0 or after > 0
    again = P.decay_attention_backward(g, q, k, v, log_decay, starts=starts, state=first, grad_final=dafter, grad_state=True)
    assert all(torch.equal(x, y) for x, y in zip(again, want))


def test_segments_taken_and_not_begun():
    """256 segments of 8 chunks: with 148 CTAs, or somewhat fewer, the second ones are taken ahead while the first are walked over, and the copies stop
    behind the first chunk.  No row is left as it was."""
    q, k, v, _, _, log_decay, _, _ = make([1000] * 4, 64, 64, 64, 64, torch.bfloat16, packed=False, seed=27)
    out = torch.full_like(q, SEVEN)
    assert lost(0, (q, k, v, out, None, None, None), (log_decay, None), (None,) * 4, (4, 1000, 4, 64, 64, 64, 64), q.dtype, 1) == B.PCR_OK
    torch.cuda.synchronize()
    want, _ = P.decay_attention(q, k, v, log_decay)
    assert whole_or_lost(out, want, "out") == 4 * 64 * 1000


def test_rows_of_no_sequence_stay_zero():
    """They are written with the first segments' rows, also where those are lost."""
    q, k, v, _, _, log_decay, _, _ = make([600], 2, 1, 64, 64, torch.bfloat16, seed=25)
    starts = torch.tensor([9, 300, 555], dtype=torch.int32, device=DEV)
    out = torch.full_like(q, SEVEN)
    args = M._DECAY_ARGS.pack(*(x for t in (q, k, v, out, None, None, None) for x in (M._NO_ROWS if t is None else M._rows(t))), *map(M._at, (log_decay, starts)), *map(M._at, (None,) * 4),
                              1, 600, 2, 2, 1, 64, 64, M._CODES[q.dtype], B.PCR_DECAY_ZERO_TAIL)
    scratch = torch.full((1 << 20,), SEVEN, device=DEV)
    assert B.lib().pcr_selftest_decay_waits(args, 0, scratch.data_ptr(), 0, torch.cuda.current_stream().cuda_stream) == B.PCR_OK
    torch.cuda.synchronize()
    assert not out[:9].any() and not out[555:].any() and out[9:555].isnan().all()


def test_only_where_there_are_such_waits():
    q, k, v, _, _, log_decay, _, _ = make([64], 2, 2, 64, 64, torch.float32, packed=False)
    assert lost(0, (q, k, v, torch.empty_like(q), None, None, None), (log_decay, None), (None,) * 4, (1, 64, 1, 2, 2, 64, 64), torch.float32, 0) == B.PCR_E_ARG
    assert B.lib().pcr_selftest_decay_waits(None, 0, None, C.c_uint32(0), None) == B.PCR_E_ARG


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [16, 40, 128])
def test_short_sequences_one_behind_the_other(size, dtype):
    """Segments of a chunk with rows to clear each, many to a CTA, as fast as they come: no wait runs out (after two seconds there would be NaN)."""
    lengths = [127, 5, 61, 1, 127, 127, 2, 100, 13, 126, 90, 1, 127, 33, 120, 7] * 2
    q, k, v, g, starts, log_decay, _, _ = make(lengths, 16, 16, size, size, dtype, seed=29)
    want = (P.decay_attention(q, k, v, log_decay, starts=starts)[0], *P.decay_attention_backward(g, q, k, v, log_decay, starts=starts)[:3])
    for x, y in zip(want, (P.decay_attention(q.float(), k.float(), v.float(), log_decay, starts=starts)[0],
                           *P.decay_attention_backward(g.float(), q.float(), k.float(), v.float(), log_decay, starts=starts)[:3])):
        assert float((x.float() - y).norm() / y.norm()) < torch.finfo(dtype).eps
    for _ in range(150):
        got = (P.decay_attention(q, k, v, log_decay, starts=starts)[0], *P.decay_attention_backward(g, q, k, v, log_decay, starts=starts)[:3])
        assert all(torch.equal(x, y) for x, y in zip(got, want))
