"""Softmax weights of 16 bits: one key that takes most of a row beside very many that share the rest.

Weights of F16 are held at 2^11 times their size relative to the row's largest, so that they are subnormal only below
2^-25 of it, and rounded to steps of 2^-35 there: a key that is seen adds an error of 2^-36 of its value at most to what
`attend_bound` allows, relative to a sum of weights of at least 1.
"""
import pytest
import torch

from tests.clear_util import Cache, attend_bound, attend_ref, close, gen

pytestmark = pytest.mark.gpu


def sink(lens, heads, kv_heads, dim, dtype, gap, at, seed):
    """Every query's score with key `at` of a sequence is `gap`, with the others 0; the value of that key is 0, others lie in [0.5, 1.5]."""
    c = Cache(lens, heads, kv_heads, dim, 64, dtype, seed)
    c.q.zero_()
    c.q[..., 0] = 1
    c.k.zero_()
    c.v.copy_(0.5 + torch.rand(c.v.shape, generator=gen(seed), device="cuda"))
    for b, (n, kv) in enumerate(lens):
        p = min(at, kv - n)
        c.k[int(c.table[b, p // 64]), :, p % 64, 0] = gap
        c.v[int(c.table[b, p // 64]), :, p % 64] = 0
    return c


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("gap", [10.0, 14.0, 16.0, 17.0, 17.5, 20.0])
@pytest.mark.parametrize("shape", [([(1, 131072), (3, 70000)], 4, 2, 64), ([(1, 131072)], 2, 1, 256), ([(600, 60000)], 8, 1, 128), ([(600, 60000)], 8, 1, 64),
                                   ([(300, 20000)], 8, 1, 256), ([(2, 700), (1, 9000)], 4, 4, 128)])
def test_one_key_against_many(shape, gap, dtype):
    from paper_2604_09975_amd import clear as K
    for at in (0, 5000):
        c = sink(*shape, dtype, gap, at, int(gap))
        lse = torch.empty(c.total, c.heads, device="cuda")
        out = K.ckks_clear_attend(c.q, *c.args(), scale=1.0, lse=lse)
        want, wl, mass = attend_ref(c, scale=1.0)
        bound = attend_bound(c, want, mass)
        if dtype is torch.float16:
            bound = bound + 2.0**-36 * 1.5 * max(kv for _, kv in shape[0])
        close(out, want, bound, "out")
        close(lse, wl, 2.0**-13 * (1 + wl.abs()), "lse")


def test_weights_stay_in_range_as_scores_rise():
    """Scores that rise by 3.9 powers of two from tile to tile, just what the maximum may lag behind, and by more."""
    from paper_2604_09975_amd import clear as K
    for step in (2.0, 3.9, 4.1, 7.9):
        c = Cache([(1, 640), (40, 640)], 4, 2, 128, 64, torch.float16, 3)
        c.q.zero_()
        c.q[..., 0] = 1
        c.k.zero_()
        for b in range(2):
            for p in range(640):
                c.k[int(c.table[b, p // 64]), :, p % 64, 0] = step * 0.6931 * (p // 32)
        out = K.ckks_clear_attend(c.q, *c.args(), scale=1.0)
        want, _, mass = attend_ref(c, scale=1.0)
        close(out, want, attend_bound(c, want, mass))
