"""Calls on pages of 8 bits that the documentation allows and that are easily forgotten: no pages at all, a table of no width, rows in no
sequence, two rows of one array for outputs, very many tokens, widths that no form was made for."""
import math

import pytest
import torch

from tests.clear_util import TYPES, U, attend_bound, attend_ref, close, gen, randn
from tests.packed_util import FORMATS, PackedCache, pack_ref, values
from tests.test_gpu_clear_packed_attend import check as check_attend
from tests.test_gpu_clear_packed_cache import check as check_append, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [16, 72, 128])
def test_no_pages_and_no_table(dim, dtype):
    from paper_2604_09975_amd import clear as K
    g, dtype = gen(1), TYPES[dtype]
    for n_pages, width in ((0, 3), (0, 0), (2, 0)):
        codes = [torch.zeros(n_pages, 2, 32, dim, dtype=torch.int8, device="cuda") for _ in range(2)]
        power = [torch.zeros(n_pages, 2, 32, -(-dim // 32), dtype=torch.uint8, device="cuda") for _ in range(2)]
        table = torch.zeros(2, width, dtype=torch.int32, device="cuda")
        start, kv = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1, 4], [70, 3]))
        q, k, v = (randn(g, 4, h, dim, dtype=dtype) for h in (4, 2, 2))
        assert torch.equal(K.ckks_clear_packed_append(k, v, *codes, *power, table, start, kv, q=q), q)
        out = K.ckks_clear_packed_attend(q, *codes, *power, table, start, kv)
        assert not out.any()  # zeros for keys and values, or no key
        got = K.ckks_clear_packed_read(*codes, *power, table, start, kv, 4, dtype)
        assert not got[0].any() and not got[1].any()
        assert not any(x.any() for x in codes + power)


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [24, 40, 48, 56, 72, 96, 112, 120, 144, 248])
def test_every_width(dim, dtype, form):
    c = PackedCache([(1, 70), (3, 3), (40, 133)], 6, 2, dim, 32, TYPES[dtype], dim, FORMATS[form])
    check_append(c, rows_of(c, dim), norms=(1 + 0.1 * randn(gen(1), dim), 1 + 0.1 * randn(gen(2), dim)))
    check_attend(c)
    check_attend(c, window=33)


def test_rows_in_no_sequence_are_left_as_they_were():
    from paper_2604_09975_amd import clear as K
    for n, heads in ((1, 4), (60, 32)):
        c = PackedCache([(n, 200), (n, 90)], heads, 2, 64, 16, torch.bfloat16, 4)
        q = torch.cat((c.q, c.q[:7]))
        out = torch.full_like(q, 7.0)
        lse = torch.full((q.shape[0], heads), 7.0, device="cuda")
        K.ckks_clear_packed_attend(q, *c.args(), out=out, lse=lse)
        assert (out[2 * n:] == 7).all() and (lse[2 * n:] == 7).all()
        want, _, mass = attend_ref(c)
        close(out[:2 * n], want, attend_bound(c, want, mass))


def test_more_tokens_than_a_grid_has_columns():
    """80000 tokens: their places, rows that are read back, and a few of them against 64 bits."""
    from paper_2604_09975_amd import clear as K
    n, page = 80000, 64
    g = gen(3)
    codes = [torch.zeros(n // page, 1, page, 32, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    power = [torch.zeros(n // page, 1, page, 1, dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = torch.randperm(n // page, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()[None]
    start, kv = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [n]))
    k, v = (randn(g, n, 1, 32) for _ in range(2))
    K.ckks_clear_packed_append(k, v, *codes, *power, table, start, kv)
    got = K.ckks_clear_packed_read(*codes, *power, table, start, kv, n)
    for x, y in zip((k, v), got):
        assert torch.equal(y.double(), pack_ref(x.double(), torch.float8_e4m3fn)[0])
    held = values(codes[0], power[0])[table[0].long()].reshape(n, 1, 32)
    assert torch.equal(held, got[0].double())


def test_the_same_page_twice_in_a_table_is_read_twice():
    from paper_2604_09975_amd import clear as K
    for n in (1, 40):
        c = PackedCache([(n, 96)], 4, 2, 64, 32, torch.float16, 9)
        c.table[0, 2] = c.page_table[0, 2] = int(c.table[0, 0])
        check_attend(c)
        k, _ = K.ckks_clear_packed_read(*c.codes, *c.power, c.page_table, torch.tensor([0, 96], dtype=torch.int32, device="cuda"), c.kv_len, 96)
        assert torch.equal(k[:32], k[64:])


def test_lengths_that_no_sequence_can_have():
    """Negative lengths and starts that do not rise: nothing outside the arrays is touched, sequences that are whole come out right."""
    from paper_2604_09975_amd import clear as K
    c = PackedCache([(2, 50), (1, 30), (3, 80)], 4, 2, 64, 16, torch.bfloat16, 11)
    want = K.ckks_clear_packed_attend(c.q, *c.args())
    bad = c.kv_len.clone()
    bad[1] = -5
    got = K.ckks_clear_packed_attend(c.q, *c.codes, *c.power, c.page_table, c.q_start, bad)
    assert torch.equal(got[:2], want[:2]) and torch.equal(got[3:], want[3:]) and not got[2].any()
    for start in ([5, 1, 3, 6], [-2**31, 2, 3, 2**31 - 1], [0, 6, 2, 6]):
        s = torch.tensor(start, dtype=torch.int32, device="cuda")
        K.ckks_clear_packed_attend(c.q, *c.codes, *c.power, c.page_table, s, c.kv_len)
        K.ckks_clear_packed_read(*c.codes, *c.power, c.page_table, s, c.kv_len, 6)
    torch.cuda.synchronize()
    assert torch.equal(want, K.ckks_clear_packed_attend(c.q, *c.args()))


def test_scores_without_end_and_scale():
    """A single key: its value whatever the score; queries of infinity and NaN give NaN to their own rows alone."""
    from paper_2604_09975_amd import clear as K
    for dtype in TYPES.values():
        c = PackedCache([(1, 1), (2, 40)], 4, 2, 64, 16, dtype, 12)
        c.q[0] *= 50
        out = check_attend(c)
        v = c.keys(0, "v")[0]
        v = v.repeat_interleave(2, 0)
        # w v / w: the products of w's parts, their sum, the quotient and its product are rounded in 32 bits, the result once more
        close(out[0], v, (U[dtype] + 6 * 2.0**-24) * v.abs())
        c.q[1, 2, 5] = math.nan
        c.q[2, 0, 7] = math.inf
        got = K.ckks_clear_packed_attend(c.q, *c.args())
        assert torch.isnan(got[1, 2]).all() and not torch.isfinite(got[2, 0]).any()
        got[1, 2] = got[2, 0] = 0
        ref = out.clone()
        ref[1, 2] = ref[2, 0] = 0
        assert torch.equal(got, ref)
