"""The decode step's operators at the edges of their number types: how many bits what lies between their two products has,
infinite values and weights, sums and scores near the largest number.  Expected results are the formulas', in 64 bits."""
import numpy as np
import pytest
import torch

import decode_step_reference as R
from paper_2511_10676_amd import binding as B
from test_gpu_decode_step import _cache, _i32, _np, _pages, _storage, _to

pytestmark = pytest.mark.gpu


def _two_parts(x):
    """x as the sum of two bf16 numbers: the nearest, and the nearest to what is left."""
    high = _storage(x, "bf16").astype(np.float64)
    return high, _storage(x - high, "bf16").astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,where", [(3, (0, 1, 2)), (40, (5, 6, 7)), (40, (5, 38, 17)), (3000, (100, 1700, 2800)), (3000, (1700, 1701, 1702)), (20000, (19999, 0, 7777))])
def test_attend_multiplies_probabilities_of_32_bits(n, where, dtype):
    """Head h looks at three positions, with weights in the ratio 1 : e : e (e = exp(-s_h), s_h < 1); dimension h of their
    values is 1, -v1, -v2 with v1 + v2 close to 1 / e, so that the sum all but cancels and shows what the weights were off by.
    Of the sum, whose terms are 1 at most: e is off by its argument's rounding (2 U) and the exponential's (2 U), the products
    of bf16 numbers with parts of e are exact, and about 8 sums of terms up to 1 round (U each; their join over chunks 4 more):
    16 U.  A weight of 16 bits is off by up to 64 U."""
    H, G, D = 1, 16, 16
    kp, vp, table = _cache(np.random.default_rng(n), [n], H, D, D, 16, dtype)
    g = np.random.default_rng(40)
    s = _storage(g.uniform(0.2, 0.95, G), "bf16").astype(np.float64)       # exact in both types
    e = np.exp(-s)
    q = np.zeros((1, G, D))
    q[0, :, 0], q[0, :, 1] = s, 256.0
    pos = np.array(where)
    page, slot = table[0, np.arange(n) // 16], np.arange(n) % 16
    kp[page, 0, slot], vp[page, 0, slot] = 0.0, 0.0
    kp[page, 0, slot, 1] = -4.0                            # everyone else: a score of -1024, a weight of 0
    kp[page[pos], 0, slot[pos], 1] = 0.0
    kp[page[pos[1:]], 0, slot[pos[1:]], 0] = -1.0          # scores 0, -s, -s
    high, low = _two_parts(1.0 / e)
    vp[page[pos[0]], 0, slot[pos[0]]] = 1.0
    vp[page[pos[1]], 0, slot[pos[1]]], vp[page[pos[2]], 0, slot[pos[2]]] = -high, -low
    got = B.attend(_to(q, dtype), _pages(kp, dtype, "heads"), _pages(vp, dtype, "heads"), _i32(table), _i32([n]), scale=1.0)
    torch.cuda.synchronize()
    want = (1.0 - e[:, None] * (high + low)[None]) / (1.0 + 2.0 * e[:, None])          # [head, dimension]
    size = np.maximum(1.0, e[:, None] * np.abs(high + low)[None])
    tol = 16 * R.U * size / (1.0 + 2.0 * e[:, None]) + (R.BF16 if dtype == "bf16" else 4 * R.U) * np.abs(want)
    off = np.abs(_np(got.out)[0].astype(np.float64) - want)
    assert (off <= tol).all(), (off / tol).max()
