"""Infinities and NaN in linear attention with a decay: what they make of memories and of the outputs behind them is what the recurrence
S = f S + k v^T makes of them, whichever kernel takes the call (16-bit operands go through tensor cores in parts, where inf - inf would be no number)."""
import pytest
import torch

import paper_1911_00472_b200 as P
from test_gpu_decay import DEV, DTYPES

pytestmark = pytest.mark.gpu


def recurrence(q, k, v, log_decay, lengths, reverse=False):
    """(outputs, memories behind) token by token in 64 bits; keys, queries and values of as many heads."""
    f = log_decay.double().exp()[:, None, None]
    out, after, at = torch.zeros(q.shape[0], q.shape[1], v.shape[-1], device=DEV, dtype=torch.float64), [], 0
    for n in lengths:
        s = torch.zeros(q.shape[1], q.shape[2], v.shape[2], device=DEV, dtype=torch.float64)
        for t in range(at + n - 1, at - 1, -1) if reverse else range(at, at + n):
            s = f * s + k[t].double()[:, :, None] * v[t].double()[:, None, :]
            out[t] = (q[t].double()[:, :, None] * s).sum(1)
        after.append(s)
        at += n
    return out, torch.stack(after)


def alike(got, want, what):
    """The same infinities, the same NaN, finite elsewhere."""
    assert torch.equal(got.isnan(), want.isnan()), (what, "NaN", int(got.isnan().sum()), int(want.isnan().sum()))
    assert torch.equal(got.isinf(), want.isinf()), (what, "infinities")
    bad = want.isinf()
    assert torch.equal(got[bad].sign().double(), want[bad].sign()), (what, "signs")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [64, 128, 40, 24])
@pytest.mark.parametrize("lengths", [[300, 77], [1500, 200]], ids=str)
@pytest.mark.parametrize("which", ["key", "value"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_one_element(value, which, lengths, size, dtype):
    """One element of a key, which reaches a row of the memory, or of a value, which reaches a column; queries and keys that are positive, so
    that infinities meet none of the other sign."""
    n = sum(lengths)
    g = torch.Generator(device=DEV).manual_seed(size + n)
    q, k = (torch.rand(n, 2, size, device=DEV, generator=g).add_(0.25).to(dtype) for _ in range(2))
    v = torch.randn(n, 2, size, device=DEV, generator=g).to(dtype)
    v[v == 0] = 1
    at = 150
    (k if which == "key" else v)[at, 1, size - 3] = value
    log_decay = torch.tensor([-0.02, -0.005], device=DEV)
    starts = torch.tensor([0, lengths[0], n], dtype=torch.int32, device=DEV)
    out, after = P.decay_attention(q, k, v, log_decay, starts=starts, final=True)
    want, memory = recurrence(q, k, v, log_decay, lengths)
    alike(after, memory, "memory")
    alike(out, want, "out")
    assert torch.isfinite(out[:at]).all() and torch.isfinite(out[lengths[0]:]).all() and torch.isfinite(after[1]).all()
    fine = torch.isfinite(memory)                                    # what is finite beside them is as right as ever
    assert torch.allclose(after[fine].double(), memory[fine], rtol=1e-4, atol=1e-4)
    fine = torch.isfinite(want)
    assert torch.allclose(out[fine].double(), want[fine], rtol=0, atol=4 * torch.finfo(dtype).eps * float(want[fine].abs().max()) + 1e-4)
    # the same walk from the other end: gradients of the memory before, whose "keys" are queries and whose "values" the outputs' gradients
    x = q.clone()
    gr = v.clone()
    (x if which == "key" else gr)[at, 1, size - 5] = value
    k = torch.where(torch.isfinite(k), k, 1.0)
    v = torch.where(torch.isfinite(v), v, 1.0)
    _, _, dv, before = P.decay_attention_backward(gr, x, k, v, log_decay, starts=starts, grad_state=True)
    want, memory = recurrence(k, x, gr, log_decay, lengths, True)
    alike(before, memory, "dstate")
    alike(dv, want, "dv")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [64, 128])
def test_all_tokens_are_no_numbers(size, dtype):
    """Everything is NaN, and soon: what is no number is not added up again."""
    q, k, v = (torch.full((4096, 2, size), float("nan"), device=DEV, dtype=dtype) for _ in range(3))
    log_decay = torch.tensor([-0.02, -0.005], device=DEV)
    out, after = P.decay_attention(q[None], k[None], v[None], log_decay, final=True)
    assert out.isnan().all() and after.isnan().all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinite_memories_to_begin_with(dtype):
    n, size = 400, 64
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k = (torch.rand(n, 2, size, device=DEV, generator=g).add_(0.25).to(dtype) for _ in range(2))
    v = torch.randn(n, 2, size, device=DEV, generator=g).to(dtype)
    first = torch.zeros(1, 2, size, size, device=DEV)
    first[0, 0, 5, 7], first[0, 1, 9, 11] = float("inf"), float("-inf")
    out, after = P.decay_attention(q, k, v, torch.tensor([-0.02, -0.005], device=DEV), starts=torch.tensor([0, n], dtype=torch.int32, device=DEV), state=first, final=True)
    bad = torch.zeros_like(after, dtype=torch.bool)
    bad[0, 0, 5, 7] = bad[0, 1, 9, 11] = True
    assert torch.equal(after.isinf(), bad) and not after.isnan().any() and after[0, 0, 5, 7] > 0 and after[0, 1, 9, 11] < 0
    assert (out[:, 0, 7] == float("inf")).all() and (out[:, 1, 11] == -float("inf")).all()
    out[:, 0, 7] = out[:, 1, 11] = 0
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [64, 128])
def test_memories_near_the_end_of_single_precision(size, dtype):
    """Memories of 2^125 are numbers: a query of zeros reads 0 from them, a small one what is there (2^-24 2^125 is above fp16's range, in bf16 a number)."""
    n = 200
    q = torch.zeros(1, n, 2, size, device=DEV, dtype=dtype)
    q[:, 150:, :, 3] = 2.0 ** -24
    k = torch.zeros_like(q)
    v = torch.ones_like(q)
    first = torch.full((1, 2, size, size), 2.0 ** 125, device=DEV)
    out, after = P.decay_attention(q, k, v, torch.zeros(2, device=DEV), state=first, final=True)
    assert not out[:, :150].any() and torch.equal(after, first)
    assert (out[:, 150:] == (float("inf") if dtype == torch.float16 else 2.0 ** 101)).all()
