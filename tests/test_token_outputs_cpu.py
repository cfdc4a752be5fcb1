"""Outputs of the token operators that share memory with what the same call reads or writes are refused.  Calls that would be
accepted are not made here: the addresses are made up."""
import ctypes as C
import itertools
import os
import random
import subprocess

import pytest

import paper_1911_00472_b200
from paper_1911_00472_b200 import binding as B
from test_tokens_cpu import TurnArgs

E = B.PCR_E_ARG
CSRC = os.path.join(os.path.dirname(paper_1911_00472_b200.__file__), "csrc")

SHIM = r"""
#include "pcr_spans.h"
extern "C" int shared(const int64_t* a, const int64_t* b) {       // address, bytes, three steps, three counts
    auto span = [](const int64_t* s) {
        const int64_t step[3] = {s[2], s[3], s[4]};
        return pcr::span_of((const void*)s[0], step, s[5], s[6], s[7], s[1], 1);
    };
    return pcr::share_memory(span(a), span(b));
}
"""


@pytest.fixture(scope="module")
def shared(tmp_path_factory):
    at = tmp_path_factory.mktemp("spans")
    (at / "shim.cc").write_text(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, "-o", str(at / "shim.so"), str(at / "shim.cc")])
    fn = C.CDLL(str(at / "shim.so")).shared
    return lambda a, b: bool(fn((C.c_int64 * 8)(*a), (C.c_int64 * 8)(*b)))


def bytes_of(span):
    at, row, *rest = span
    return {at + sum(s * i for s, i in zip(rest[:3], where)) + j for where in itertools.product(*(range(n) for n in rest[3:])) for j in range(row)}


def test_spans_against_sets_of_bytes(shared):
    rng = random.Random(7)
    seen = {True: 0, False: 0}
    for _ in range(6000):
        if rng.random() < 0.5:                  # slices of one buffer: steps alike
            row = rng.choice([1, 2, 4])
            steps = [rng.choice([row * 8, row * 16, 48]), rng.choice([row * 3, row * 8]), rng.choice([0, row, row * 2])]
            spans = [(1000 + rng.randint(0, 60), row, *steps, *(rng.randint(0 if rng.random() < 0.05 else 1, 4) for _ in range(3))) for _ in range(2)]
        else:
            spans = [(1000 + rng.randint(0, 90), rng.randint(1, 5), *(rng.randint(-30, 30) for _ in range(3)), *(rng.randint(1, 4) for _ in range(3))) for _ in range(2)]
        want = bool(bytes_of(spans[0]) & bytes_of(spans[1]))
        assert shared(*spans) == want, spans
        seen[want] += 1
    assert min(seen.values()) > 500


def test_spans_of_large_buffers(shared):
    """Queries, keys and values side by side in one projection's output, heads before tokens, far strides."""
    row, far = 128 * 2, 1 << 45
    for steps, n in (((32768 * 12 * row, 12 * row, row), (4, 32768)), ((12 * 32768 * row, row, 32768 * row), (4, 32768)), ((far, 1 << 33, row), (65535, 4096))):
        part = lambda first, heads: ((1 << 46) + first * steps[2], row, *steps, *n, heads)  # noqa: E731
        assert not shared(part(0, 8), part(8, 2)) and not shared(part(8, 2), part(10, 2)) and not shared(part(10, 2), part(0, 8))
        assert shared(part(0, 9), part(8, 2)) and shared(part(0, 8), part(0, 8)) and shared(part(3, 1), part(0, 12))


def good():
    """Arguments without shared memory (never launched as they are)."""
    a = TurnArgs()
    for i, h in enumerate((a.q, a.k)):
        base = (1 + i) << 20
        h.x, h.y, h.dy, h.weight, h.dweight, h.heads = base, base + (1 << 16), base + (2 << 16), base + (3 << 16), base + (4 << 16), 2
        for s in (h.x_stride, h.y_stride, h.dy_stride):
            s[0], s[1], s[2] = 5 * 128, 128, 64
    a.positions, a.inv_freq, a.axes = 3 << 20, 4 << 20, 5 << 20
    a.position_stride[:] = (15, 5, 1)
    a.batch, a.tokens, a.n_axes, a.head_dim, a.rot_dim = 3, 5, 3, 64, 64
    a.dtype, a.freq_dtype, a.weight_dtype, a.eps = B.PCR_BF16, B.PCR_F64, B.PCR_F32, 1e-6
    return a


SCRATCH = 6 << 20
ROW = 2 * 64                                          # bytes of a head


def q_y_on(name):
    def change(a):
        a.q.y = getattr(a.k, name[2:]) if name.startswith("k.") else getattr(a.q, name[2:]) if name.startswith("q.") else getattr(a, name)
    return change


def nudged(a):
    a.q.y = a.q.x + 2                                 # its own operand, an element further on


def other_strides(a):
    a.q.y = a.q.x
    a.q.y_stride[1], a.q.y_stride[2] = 64, 5 * 64     # heads before tokens in the same memory


def one_head_further(a):
    a.k.x_stride[:] = a.k.y_stride[:] = a.q.x_stride[:] = a.q.y_stride[:] = (5 * 256, 256, 64)
    a.k.y = a.q.x + ROW


@pytest.mark.parametrize("change", [q_y_on("k.x"), q_y_on("k.y"), q_y_on("positions"), q_y_on("inv_freq"), q_y_on("axes"), nudged, other_strides, one_head_further],
                         ids=["k.x", "k.y", "positions", "inv_freq", "axes", "nudged", "other strides", "one head further"])
def test_refused_by_every_call(change):
    a = good()
    change(a)
    L, raw = B.lib(), bytes(a)
    assert (L.pcr_rotate(raw, None), L.pcr_norm_rotate(raw, None), L.pcr_norm_rotate_backward(raw, SCRATCH, None)) == (E, E, E)


@pytest.mark.parametrize("name", ["q.weight", "k.weight"])
def test_refused_by_the_norms(name):
    a = good()
    q_y_on(name)(a)
    L, raw = B.lib(), bytes(a)
    assert (L.pcr_norm_rotate(raw, None), L.pcr_norm_rotate_backward(raw, SCRATCH, None)) == (E, E)


@pytest.mark.parametrize("name", ["k.dy", "q.dweight", "k.dweight"])
def test_refused_by_the_backward_pass(name):
    a = good()
    q_y_on(name)(a)
    assert B.lib().pcr_norm_rotate_backward(bytes(a), SCRATCH, None) == E


def test_one_gradient_for_two_weights_and_scratch_that_is_used_already():
    L = B.lib()
    a = good()
    a.q.dweight = a.k.dweight
    assert L.pcr_norm_rotate_backward(bytes(a), SCRATCH, None) == E
    a = good()
    for at in (a.q.x, a.k.y, a.k.dy, a.q.weight, a.k.dweight, a.positions, a.inv_freq, a.axes, a.q.dweight - 4):
        assert L.pcr_norm_rotate_backward(bytes(a), at, None) == E


def test_patch_tokens_over_what_they_are_made_of():
    import struct
    call = B.lib().pcr_patch_tokens
    m, s = struct.pack("3f", 0.5, 0.5, 0.5), struct.pack("3f", 0.2, 0.2, 0.2)
    rgb, images, index, out = 1 << 20, 2 << 20, 3 << 20, 10 * 3 * 14 * 14 * 2         # (addresses, and the bytes of the output)
    for at in (rgb, rgb + 996, images - out + 2, images + 158, index + 78, index - 2):
        assert call(rgb, 1000, images, 2, index, 10, 14, 2, m, s, B.PCR_BF16, at, None) == E, hex(at)


def test_positions_over_what_they_are_made_of():
    call = B.lib().pcr_token_positions
    segments, after, scratch = 1 << 20, 2 << 20, 3 << 20
    n, few, many = 100, 3, 20000
    for at in (segments, segments + 44, segments - 8 * n - 400 + 4, after, after + 4, after - 4 * n):           # rows of 400 bytes, 400 bytes apart
        assert call(segments, few, n, 2, 1, 1, 0, at, n, after, None, None) == E, hex(at)
    assert call(segments, few, n, 2, 1, 1, 0, 4 << 20, n, segments + 16, None, None) == E                       # the sequences' ends over a segment
    for at in (segments, after, 4 << 20):
        assert call(segments, many, n, 2, 1, 1, 0, 4 << 20, n, after, at, None) == E
    assert call(segments, many, n, 2, 1, 1, 0, scratch + 8, n, after, scratch, None) == E
