"""Shared-prefix decode on the GPU: the roundings of the weights cancel in what all values have in common."""
import math

import pytest
import torch

from tests.test_gpu_decode_shared import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,D,bs", [(8, 8, 64, 16), (16, 8, 128, 16), (16, 4, 128, 32), (8, 1, 128, 16)])
def test_a_value_that_all_keys_have_comes_out_exactly(Hq, Hkv, D, bs):
    """Weights are rounded to bf16 once, the same ones for the products and the denominator.  One key in 64 has the highest
    score, so that every piece has its maximum; the others weigh 0.5019, which bf16 rounds to 0.5: over unrounded weights the
    quotient would be (1 + 63 * 0.5) / (1 + 63 * 0.5019) = 0.9963.  With rounded ones both sums are exact, and quotient and merge
    are off by a few 2^-23, far from the half step of 2^-9 below 1."""
    b = Batch(Hq, Hkv, D, bs, sizes=[5, 2], prefix=[1500, 320], lens=[1501, 1564, 1700, 1536, 2000, 321, 900, 70], loose=1)
    b.q.zero_()
    b.q[..., 0] = 1
    b.k, b.v = torch.where(b.k.isnan(), b.k, 0), torch.where(b.v.isnan(), b.v, 1)
    for s in range(b.B):
        b.k[b.table[s, :-(-b.n[s] // bs):64 // bs].long(), :, 0, 0] = 1
    for ws in (None, b.workspace(512, small=True)):
        assert bool((b.run(-math.log(0.5019), ws=ws) == 1).all())
