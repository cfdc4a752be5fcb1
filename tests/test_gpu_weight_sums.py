"""Gradients of the norms' weights over many rows, on data where a row that is left out shows.

With g = the turned, normed x, what a row adds to an element is the square of its normed value (but for g's rounding, which the
reference sees too): nothing cancels, and dw grows with the rows.  Tolerance, u = 2^-24, in units of u times the sum of
(|a| + |b|) |v| (a, b: the pair of g that makes d; v = x r): a turned element is off by 16 units and r by 32 (as in the tests of
queries and keys), their product by 2.  The additions that lie between a term and the result: a lane's own rows, fewer than 60
at these sizes on 148 SMs (the fewest lanes at a time: 333 CTAs of 8 rows for 12001 tokens of 6 heads, 5 rounds of 6), a warp's up to
32 rows, 4 warps, and of the rows of partial sums, 1184 at most, every 32nd and then 32: 37 + 32.  60 + 32 + 4 + 69 = 165."""
import pytest
import torch

import paper_1911_00472_b200 as P
from test_gpu_heads import DTYPES, U, angle_of, make, turned

pytestmark = pytest.mark.gpu


def check_sums(x, g, dw, angle, interleaved, weight):
    x, g = x.double(), g.double()
    d, size = turned(g, -angle, interleaved)
    v = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    want, slack = (d * v).sum((0, 1, 2)), (16 + 32 + 2 + 165) * U * (size * v).abs().sum((0, 1, 2))
    assert bool((slack * 10000 <= want).all())                  # one in ten thousand rows left out would show
    off = (dw.double() - want).abs()
    assert dw.dtype == torch.float32 and bool((off <= slack + U * want).all()), float((off / slack).max())


# tokens: one round and a half, more than two, more than four of the CTAs that take queries or keys
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("layout", ["packed", "shifted"])
@pytest.mark.parametrize("size", [128, 72, 36])
@pytest.mark.parametrize("batch,tokens", [(2, 4099), (1, 12001), (7, 643)])
def test_no_row_is_lost(batch, tokens, size, layout, dtype):
    q, k, positions, inv_freq, axes, wq, wk = make((batch, tokens, 6, 2, size, size), dtype, layout, weight_dtype=torch.float32)
    angle, next_ = angle_of(positions, inv_freq, axes), tokens == 643
    grads = [turned(x.double() / (x.double().square().mean(-1, keepdim=True) + 1e-6).sqrt(), angle, next_)[0].to(dtype) for x in (q, k)]
    got = P.norm_rotate_backward(*grads, q, k, wq, wk, positions, inv_freq, axes, interleaved=next_)
    check_sums(q, grads[0], got[2], angle, next_, wq)
    check_sums(k, grads[1], got[3], angle, next_, wk)
