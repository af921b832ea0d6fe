"""The weights of the prefix attention keep fp32's bits: outputs whose terms cancel show it, where an ordinary output's own rounding hides it.

Three tokens: the first has weight 1 and value 1, the others weights w2 + w3 = 1 up to about 1e-5 and value -1, so out = (1 - w2 - w3) / 2
is rounded to bf16 by 2^-8 of almost nothing.  What is left, relative to sum p|v| = 1: |scores| of at most 3 in units of log2, two
roundings (2^-24 each) of scale and product, one of the exponential (2^-23): 4e-7 of each weight, half of it in the output;
the sums' own roundings, twelve terms of at most 1 with 2^-24 each, or 2^-23 where an addition cuts off: 7e-7 of l = 2 at most.
Bound: 2^-8 |ref| + 2^-20.  (Weights rounded to sixteen bits leave up to 2^-18 of each.)"""
import math

import pytest
import torch

import paper_2505_18573_amd as e3
from tests.test_prefix_attention import BF16, DEV, FP8, Step


class Cancelling(Step):
    def fill(self, pages, n, g):
        if n == 0:
            return super().fill(pages, n, g)
        k, v = torch.zeros((2, n, self.H, self.D), dtype=BF16)
        k[1, :, 0] = 1.0
        k[2, :, 1] = k[2, :, 2] = 1.0
        v[0], v[1:] = 1.0, -1.0
        at = torch.arange(n)
        slots = (pages[at // self.page] * self.page + at % self.page).to(DEV)
        e3.e3_cache_append(self.cache, k.to(DEV), v.to(DEV), slots)
        return k.double(), v.double()


def queries(shape, D, seed):
    """bf16 queries whose scores with the three keys are 0, ln w and ln (1 - w), the last one in two parts."""
    w = 0.15 + 0.7 * torch.rand(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
    q = torch.zeros((*shape, D), dtype=BF16)
    q[..., 0] = torch.log(w).to(BF16)
    rest = torch.log1p(-torch.exp(q[..., 0].double()))
    q[..., 1] = rest.to(BF16)
    q[..., 2] = (rest - q[..., 1].double()).to(BF16)
    return q


@pytest.mark.gpu
@pytest.mark.parametrize("where", ["own", "prefix"])
@pytest.mark.parametrize("cache_type", [FP8, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,R", [(1, 16), (40, 8), (9, 33)])
def test_outputs_that_cancel(where, cache_type, D, rows, R):
    # a prefix of several rows, or more than 16 query heads of a key head, is a workgroup's work, the others a wave's
    s = Cancelling([rows], [3 if where == "prefix" else 0], [3 if where == "own" else 0] * rows, 1, R, 2, D, 32, cache_type)
    s.q, s.scale = queries((rows, 1, 2 * R), D, rows + R), 1.0
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    want, size, want_lse = s.reference()
    assert float(want.abs().max()) < 1e-4 and bool(((size - 1).abs() < 1e-12).all())
    err = (out.double().cpu() - want).abs()
    assert bool((err <= 2.0 ** -8 * want.abs() + 2.0 ** -20).all()), float(err.max()) * 2 ** 20
    assert bool(((lse.double().cpu() - math.log(2.0)).abs() <= 2e-5).all()) and bool(((want_lse - math.log(2.0)).abs() < 1e-4).all())
