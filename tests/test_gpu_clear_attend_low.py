"""Single tokens and short chunks of 16-bit types: weights in two parts, so that only the result is rounded to the type."""
import math

import pytest
import torch

from tests.clear_util import TINY, U, Cache, attend_ref, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [8, 64, 104, 128, 200, 256])
def test_weights_do_not_add_their_rounding(dim, dtype):
    """The high part is at least 1 - 3 u of a weight, so that the low part's rounding is 3 u^2 of it; F16's steps end at 2^-35 of the
    largest weight.  The score's and the exponential's error of 2^-13 is that of `attend_bound`."""
    from paper_2604_09975_amd import clear as K
    u = U[dtype]
    c = Cache([(1, 3), (1, 17), (1, 40), (4, 100), (1, 700), (2, 9)], 6, 3, dim, 16, dtype, dim)
    for how in (dict(), dict(causal=False), dict(window=11)):
        out = K.ckks_clear_attend(c.q, *c.args(), **how)
        want, _, mass = attend_ref(c, **how)
        bound = u * want.abs() + (3 * u * u + 2.0**-13) * mass + TINY[dtype]
        if dtype is torch.float16:
            bound = bound + 2.0**-36 * 700 * c.v.abs().max().item()
        close(out, want, bound)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_infinite_values_that_all_see_stay_infinite(dim, dtype):
    """In tiles that every row sees in full: with neither part of a weight 0 or negative, the sum keeps its sign."""
    from paper_2604_09975_amd import clear as K
    c = Cache([(1, 300), (3, 9000), (1, 130)], 4, 2, dim, 16, dtype, dim)
    for b, p, h, e, x in ((0, 40, 0, 5, math.inf), (0, 41, 1, 6, -math.inf), (1, 70, 0, 3, math.inf), (1, 71, 0, 4, math.nan), (2, 64, 1, 2, math.inf), (2, 68, 1, 2, math.inf),
                          (2, 69, 1, 7, math.inf), (2, 33, 1, 7, -math.inf)):
        c.v[int(c.table[b, p // 16]), h, p % 16, e] = x
    out = K.ckks_clear_attend(c.q, *c.args())
    assert (out[0, :2, 5] == math.inf).all() and (out[0, 2:, 6] == -math.inf).all() and (out[1:4, :2, 3] == math.inf).all()
    assert torch.isnan(out[1:4, :2, 4]).all() and (out[4, 2:, 2] == math.inf).all() and torch.isnan(out[4, 2:, 7]).all()
    want, _, _ = attend_ref(c)
    assert torch.equal(torch.isfinite(out), torch.isfinite(want))
