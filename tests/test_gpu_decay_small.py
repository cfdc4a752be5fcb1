"""Linear attention with a decay on 16-bit operands far from size 1: keys, queries and gradients of any size that the type holds, against
the definition in 64 bits.

Tolerances are those of test_gpu_decay.py without its absolute terms (`near` there: E is the sum of the magnitudes, u = 2^-24).  What is
put into a memory is kept as hi + lo, each off by at most eps / 2 of its own size, of a factor kept alike: 2 (eps / 2)^2 <= 2^-21 E in fp16.  Below that
stands only the resolution of a chunk: its largest product lies at 2^14 or more and the last part's last bit is 2^-24, half of it 2^-25, that is 2^-39
of the largest product; a row's factor has that last bit too, times elements below 2^12 in their lifted form (2^16 where they are that large
themselves): 2^-25 2^12 / 2^14 = 2^-27 of the row's share where the factor is below 2^-3, that is of at most 2^-3 2^12 / 2^14 = 2^-5 of the
largest product.  Together below 2^-31 of the largest product for each token's |c|, and for values above 2^12 below 2^-27.  bf16 has the exponents of 32 bits.
An output is rounded to its type: half a step, half of the least number where that is larger.
"""
import pytest
import torch

import paper_1911_00472_b200 as P
from test_gpu_decay import DEV, U, walk, weights

pytestmark = pytest.mark.gpu
HALVES = [torch.float16, torch.bfloat16]


def draw(n, heads, size, scale, dtype, seed, uneven=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(n, heads, size, device=DEV, generator=g) * scale
    if uneven:                                                       # tokens of very different sizes, and none at all
        x = x * torch.exp2(torch.randint(-12, 1, (n, 1, 1), device=DEV, generator=g).float())
        x[torch.rand(n, device=DEV, generator=g) < 0.1] = 0
    return x.to(dtype)


def memory_near(got, want, M, b, c, dtype, what):
    n = len(b)
    parts = 2.0 ** -21 if dtype == torch.float16 else 2.0 ** -24
    coarse = 2.0 ** -27 if b.abs().max() >= 4096 else 2.0 ** -31
    tol = ((160 + 5 * (n // 32 + 1)) * U + parts) * M + (coarse * b.abs().max() * c.abs().sum(0) if dtype == torch.float16 else 0.0)
    assert torch.isfinite(got).all(), what
    worst = ((got.double() - want).abs() / tol.clamp(min=1e-300)).max()
    assert worst <= 1, (what, float(worst))


def output_near(got, want, E, b, c, a, dtype, size, what):
    n, eps = len(b), torch.finfo(dtype).eps
    coarse = 2.0 ** -27 if b.abs().max() >= 4096 else 2.0 ** -31
    tol = ((size + 160 + 5 * (n // 32 + 1)) * U + eps) * E + eps / 2 * want.abs() + torch.finfo(dtype).smallest_normal * eps / 2
    if dtype == torch.float16:
        tol = tol + coarse * b.abs().max() * a.abs().sum(-1, keepdim=True) * c.abs().sum(0)
    assert torch.isfinite(got).all(), what
    worst = ((got.double() - want).abs() / tol).max()
    assert worst <= 1, (what, float(worst))


RATES = torch.tensor([-0.001, -0.03, -0.5, -3.0])
SCALES = [2.0 ** -22, 2.0 ** -17, 2.0 ** -10, 1.0, 2.0 ** 12]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("uneven", [False, True])
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("n,size", [(700, 64), (300, 128), (5000, 64), (77, 40)], ids=str)
def test_memories_of_keys_and_queries_of_any_size(n, size, scale, uneven, dtype):
    """Memory behind the tokens for keys, gradient of the one before them for queries."""
    x, v = draw(n, 4, size, scale, dtype, n + size, uneven), draw(n, 4, size, 1.0, dtype, n + size + 1)
    log_decay = RATES.to(DEV)
    zero = torch.zeros(size, size, device=DEV, dtype=torch.float64)
    _, after = P.decay_attention(torch.zeros_like(x), x, v, log_decay, final=True, starts=torch.tensor([0, n], dtype=torch.int32, device=DEV))
    got = P.decay_attention_backward(v, x, torch.zeros_like(x), v, log_decay, grad_state=True, starts=torch.tensor([0, n], dtype=torch.int32, device=DEV))
    for h in range(4):
        rate, b, c = float(log_decay[h]), x[:, h].double(), v[:, h].double()
        _, _, want, M = walk(b, b, c, rate, zero)
        memory_near(after[0, h], want, M, b, c, dtype, ("memory", h))
        _, _, want, M = walk(b, b, c, rate, zero, True, False)
        f = log_decay[h].double().exp()
        memory_near(got[3][0, h], want * f, M * f, b, c, dtype, ("dstate", h))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("units", [3, 5, 44])
@pytest.mark.parametrize("n,size", [(700, 64), (400, 128)], ids=str)
def test_gradients_of_a_few_last_bits(n, size, units, dtype):
    """Gradients of the outputs that are a few times fp16's least number, all of one sign, so that what is lost of each would add up."""
    small = units * 2.0 ** -24
    q, k, v = (draw(n, 4, size, s, dtype, n + i).abs() for i, s in enumerate((2.0 ** 5, 2.0 ** 5, 2.0 ** 6)))
    g = torch.full((n, 4, size), small, device=DEV, dtype=dtype)
    log_decay = RATES.to(DEV)
    zero = torch.zeros(size, size, device=DEV, dtype=torch.float64)
    dq, dk, dv, _ = P.decay_attention_backward(g, q, k, v, log_decay)
    for h in range(4):
        rate = float(log_decay[h])
        a, b, c, o = (x[:, h].double() for x in (q, k, v, g))
        for what, got, (s, t, u), rev in (("dq", dq, (o, c, b), False), ("dk", dk, (c, o, a), True), ("dv", dv, (b, a, o), True)):
            y, E, _, _ = walk(s, t, u, rate, zero, rev, not rev)
            if y.abs().max() < torch.finfo(dtype).max / 2:
                output_near(got[:, h], y, E, t, u, s, dtype, size, (what, h))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("large,small", [(2.0 ** 13, 2.0 ** -17), (2.0 ** 11, 2.0 ** -20), (1.0, 1.0)])
@pytest.mark.parametrize("n,size", [(300, 64), (200, 128), (128, 40)], ids=str)
def test_a_fast_head_behind_large_keys(n, size, large, small, dtype):
    """Products of a row that are far above all others before they fade, and far below behind: what is left is right by itself.  A row's largest
    faded product lies at 2^-4 or more in fp16, so that half of the last bit, 2^-25, is 2^-21 of it, for each token's |c|."""
    q, k, v = draw(n, 3, size, 1.0, dtype, n), draw(n, 3, size, small, dtype, n + 1), draw(n, 3, size, 2.0 ** 10, dtype, n + 2)
    for at in (0, 1, 64, n - 1):
        k[at] = draw(1, 3, size, large, dtype, at)[0]
    log_decay = torch.tensor([-3.0, -1.0, -0.8], device=DEV)
    out, _ = P.decay_attention(q, k, v, log_decay, starts=torch.tensor([0, n], dtype=torch.int32, device=DEV))
    dq, dk, dv, _ = P.decay_attention_backward(v, q, k, v, log_decay)
    zero = torch.zeros(size, size, device=DEV, dtype=torch.float64)
    for h in range(3):
        a, b, c = (x[:, h].double() for x in (q, k, v))
        for what, got, (s, t, u), rev in (("out", out, (a, b, c), False), ("dv", dv, (b, a, c), True)):
            y, E, _, _ = walk(s, t, u, float(log_decay[h]), zero, rev, not rev)
            fine = y.abs().amax(-1) < torch.finfo(dtype).max / 2
            assert fine.any()
            eps = torch.finfo(dtype).eps
            w = weights(float(log_decay[h]), n)[0]
            most = ((s @ t.T).abs() * (w.T if rev else w)).amax(-1, keepdim=True)
            tol = ((size + 170) * U + eps) * E + 2.0 ** -21 * most * u.abs().sum(0) + eps / 2 * y.abs() + torch.finfo(dtype).smallest_normal * eps / 2
            worst = ((got[:, h].double() - y).abs() / tol)[fine].max()
            assert worst <= 1, (what, h, float(worst))
