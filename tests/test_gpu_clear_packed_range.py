"""A cache of 8 bits at the ends of the types' ranges: what is finite stays finite, on the way into the pages and out of them."""
import math

import pytest
import torch

from tests.clear_util import TINY, TYPES, U, close, gen, randn
from tests.packed_util import FORMATS, LARGEST, PackedCache, code_values, same, values

pytestmark = pytest.mark.gpu


def blocks_near_the_top(dtype, rows, seed):
    """[rows][1][32] of `dtype`: blocks whose largest entries are the type's last ones before infinity, beside others of every size."""
    g = gen(seed)
    top = torch.finfo(dtype).max
    unit = torch.rand(rows, 1, 32, generator=g, device="cuda") * 2 - 1
    x = unit.double() * torch.exp2(torch.randint(-12, 1, (rows, 1, 1), generator=g, device="cuda").double()) * top
    near = top * (1 - torch.rand(rows, 1, 8, generator=g, device="cuda").double() * 0.15)
    x[..., :8] = torch.copysign(near, x[..., :8])
    x[::3, :, 8:12] = -top
    x[1::3, :, 12:16] = top
    return x.clamp(-top, top).to(dtype)


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
def test_blocks_that_the_type_holds_stay_finite(dtype, form):
    """Each entry becomes the nearest of the codes whose value the type holds; read and appended again they are the same."""
    from paper_2604_09975_amd import clear as K
    dtype, form, n = TYPES[dtype], FORMATS[form], 300
    top = torch.finfo(dtype).max
    c, again = (PackedCache([(n, n)], 1, 1, 32, 64, dtype, 1, form) for _ in range(2))
    k, v = blocks_near_the_top(dtype, n, 2), blocks_near_the_top(dtype, n, 3)
    K.ckks_clear_packed_append(k, v, *c.args())
    got = K.ckks_clear_packed_read(*c.args(), n, dtype)
    for x, y in zip((k, v), got):
        x, y = x.double(), y.double()
        assert torch.isfinite(y).all()
        # the smallest power with which no code overflows, and of the codes within the type's range the nearest
        e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / LARGEST[form]))
        e = torch.where(x.abs().amax(-1, keepdim=True) > LARGEST[form] * torch.exp2(e), e + 1, e)
        e = torch.where(x.abs().amax(-1, keepdim=True) <= LARGEST[form] * torch.exp2(e - 1), e - 1, e)
        grid = code_values(form).cuda()
        grid = grid[torch.isfinite(grid)] * torch.exp2(e)[..., None]
        off = torch.where(grid.abs() <= top, (grid - x[..., None]).abs(), math.inf).amin(-1)
        assert torch.equal((y - x).abs(), off)
    K.ckks_clear_packed_append(*got, *again.args())
    assert all(same(a.double(), b.double()) for a, b in zip(got, K.ckks_clear_packed_read(*again.args(), n, dtype)))
    # and through attention: one key, its value
    q = torch.zeros(n, 1, 32, dtype=dtype, device="cuda")
    start, one = torch.arange(n + 1, dtype=torch.int32, device="cuda"), torch.ones(n, dtype=torch.int32, device="cuda")
    pages = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    assert torch.isfinite(K.ckks_clear_packed_attend(q, *c.args()[:4], pages, start, one)).all()


@pytest.mark.parametrize("form", FORMATS)
def test_keys_beyond_the_range_of_f16(form):
    """Normed keys may be more than F16 holds: the cache has them, and they read as infinite in F16 alone."""
    from paper_2604_09975_amd import clear as K
    c = PackedCache([(40, 40)], 1, 1, 64, 16, torch.float16, 4, FORMATS[form])
    k = randn(gen(5), 40, 1, 64, dtype=torch.float16)
    norm = torch.full((64,), 40000.0, device="cuda")
    K.ckks_clear_packed_append(k, k, *c.args(), k_norm=norm, eps=0.0)
    wide, _ = K.ckks_clear_packed_read(*c.args(), 40, torch.float32)
    narrow, _ = K.ckks_clear_packed_read(*c.args(), 40, torch.float16)
    x = k.double()
    x = x / (x * x).mean(-1, keepdim=True).sqrt() * 40000
    assert (x.abs() > 65520).any() and torch.isfinite(wide).all() and same(narrow, wide.to(torch.float16))
    assert ((wide.double() - x).abs() <= x.abs().amax(-1, keepdim=True) * 2.0**-4).all()


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_read_and_appended_again_wherever_the_type_holds_them(dtype, form):
    """Entries of every size: F32 and BF16 give the same values, F16 those that are multiples of 2^-24."""
    from paper_2604_09975_amd import clear as K
    dtype, form, n = TYPES[dtype], FORMATS[form], 400
    c, again = (PackedCache([(n, n)], 1, 1, 32, 64, dtype, 1, form) for _ in range(2))
    g = gen(6)
    low, high = (-24, 15) if dtype is torch.float16 else (-120, 125)
    x = (randn(g, n, 1, 32).double() * torch.exp2(torch.randint(low, high, (n, 1, 1), generator=g, device="cuda").double())).clamp(-60000 if dtype is torch.float16 else -3e38, 60000 if dtype is torch.float16 else 3e38).to(dtype)
    K.ckks_clear_packed_append(x, x, *c.args())
    got = K.ckks_clear_packed_read(*c.args(), n, dtype)
    c.refresh()
    K.ckks_clear_packed_append(*got, *again.args())
    twice = K.ckks_clear_packed_read(*again.args(), n, dtype)
    held = c.keys(0, "k").view(n, 1, 32)
    exact = (held * 2.0**24 == (held * 2.0**24).round()).all(-1, keepdim=True) if dtype is torch.float16 else torch.ones(n, 1, 1, dtype=torch.bool, device="cuda")
    assert exact.sum() > n // 4
    for a, b in zip(got, twice):
        assert torch.equal(a.double()[exact.expand_as(a)], held[exact.expand_as(a)]) and torch.equal(a[exact.expand_as(a)], b[exact.expand_as(a)])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,heads,dim", [([(1, 70), (2, 40)], 4, 64), ([(1, 300)], 16, 128), ([(90, 130)], 8, 128), ([(1, 50)], 2, 72)])
def test_infinite_keys(lens, heads, dim, dtype):
    """A code may stand for more than the type holds.  A key that is infinite there gives a score that is: below all others it
    has no weight, above them it leaves the row no number, as over a plain cache."""
    from paper_2604_09975_amd import clear as K
    dtype = TYPES[dtype]
    c = PackedCache(lens, heads, 2, dim, 16, dtype, 7, torch.int8)
    c.q[:, :, 5] = torch.where(torch.arange(heads, device="cuda") % 2 == 0, 1.0, -1.5).to(dtype)  # signs of the scores, by heads
    pg = int(c.table[0, 1])
    z = 127 + (10 if dtype is torch.float16 else 122)
    c.power[0][pg, 0, 3] = z
    c.codes[0][pg, 0, 3] = 0
    c.codes[0][pg, 0, 3, 5] = 100  # the 20th key of the first kv head's queries
    out = K.ckks_clear_packed_attend(c.q, *c.args())
    c.refresh()
    plain = [x.to(dtype) for x in (c.k, c.v)]
    assert torch.isinf(plain[0][pg, 0, 3, 5]) and int(torch.isinf(plain[0]).sum()) == 1
    want = K.ckks_clear_attend(c.q, *plain, c.page_table, c.q_start, c.kv_len)
    n, kv = c.lens[0]
    sees = torch.arange(kv - n, kv, device="cuda") >= 19
    first = torch.arange(heads, device="cuda") < heads // 2
    up = torch.arange(heads, device="cuda") % 2 == 0
    assert torch.isnan(want[:n][sees][:, first & up]).all() and torch.isfinite(want[:n][:, first & ~up]).all()
    # either result: weights rounded (twice U of the sum of weight times value), the result rounded once, 2^-13 of that sum for scores in 32 bits
    mass = K.ckks_clear_attend(c.q, plain[0], plain[1].abs(), c.page_table, c.q_start, c.kv_len).double()
    close(out, want.double(), 2 * (3 * U[dtype] + 2.0**-13) * 1.01 * mass.nan_to_num() + TINY[dtype])
