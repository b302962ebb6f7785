"""Attention over the paged cache against 64 bits."""
import math

import pytest
import torch

from tests.clear_util import TYPES, Cache, attend_bound, attend_ref, close, gen, randn

pytestmark = pytest.mark.gpu


def check(c, causal=True, window=0, scale=None):
    from paper_2604_09975_amd import clear as K
    lse = torch.full((c.total, c.heads), 7.0, device="cuda")
    out = K.ckks_clear_attend(c.q, *c.args(), scale=scale, causal=causal, window=window, lse=lse)
    want, wl, mass = attend_ref(c, causal, window, scale)
    close(out, want, attend_bound(c, want, mass), "out")
    # 32-bit scores of size up to about 60, and a logarithm
    close(lse, wl, torch.where(torch.isfinite(wl), 2.0**-13 * (1 + wl.abs()), 0.0), "lse")
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [8, 64, 80, 128, 136, 256])
@pytest.mark.parametrize("heads,kv_heads", [(3, 3), (8, 2)])
def test_ragged_batches(heads, kv_heads, dim, dtype):
    """Single tokens, chunks, a fresh prompt, a sequence without new tokens, lengths that end inside a tile and a page."""
    c = Cache([(1, 1), (1, 77), (5, 5), (0, 40), (37, 101), (130, 130), (3, 290)], heads, kv_heads, dim, 16, TYPES[dtype], dim + heads)
    check(c)
    check(c, causal=False)
    check(c, window=20)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_chunks_wide_enough_to_share_tiles(dim, dtype):
    """Row tiles of 128 by four waves: more than 256 of them."""
    c = Cache([(700, 1300), (513, 513), (1, 1000), (129, 640)], 32, 8, dim, 64, TYPES[dtype], dim)
    c.kv_len, c.lens = c.kv_len, c.lens
    check(c)
    check(c, window=150)


@pytest.mark.parametrize("dtype", TYPES)
def test_long_axis_split_over_blocks(dtype):
    for dim, lens in ((128, [(1, 9001), (1, 511), (2, 4100), (1, 3)]), (64, [(1, 20000)])):
        c = Cache(lens, 4, 2, dim, 64, TYPES[dtype], 11)
        check(c)
        check(c, window=3000)


def test_every_length_around_tiles_and_pages():
    for n, kv0 in ((1, 0), (2, 30), (33, 0), (31, 33)):
        c = Cache([(n, kv0 + n + i) for i in range(67)], 2, 1, 64, 16, torch.float16, n)
        check(c)


@pytest.mark.parametrize("page", [1, 5, 16, 48, 256])
@pytest.mark.parametrize("layout", ["head", "token", "both"])
def test_page_sizes_and_layouts(page, layout):
    c = Cache([(20, 333), (1, 50)], 4, 2, 64, page, torch.bfloat16, page, layout=layout)
    check(c)


def test_large_groups_and_many_heads():
    check(Cache([(3, 200), (1, 33)], 71, 1, 64, 16, torch.float16, 1))
    check(Cache([(2, 50)], 40, 40, 32, 16, torch.float32, 2))


def test_rows_without_keys():
    """A chunk that begins before the cache does: its first queries see nothing."""
    c = Cache([(10, 4), (5, 0), (1, 1)], 4, 2, 64, 16, torch.bfloat16, 3)
    out = check(c)
    assert not out[:6].any() and not out[10:15].any() and out[15].any()


def test_large_scores_and_small_scale():
    c = Cache([(40, 300), (1, 700)], 4, 2, 64, 16, torch.float32, 4)
    c.q *= 40                                  # scores of hundreds: one key takes all
    from paper_2604_09975_amd import clear as K
    out = K.ckks_clear_attend(c.q, *c.args())
    want, _, mass = attend_ref(c)
    # a score of 300 in 32 bits is off by up to 64 * 2^-24 of the sum of its products' sizes, about 2000
    close(out, want, 64 * 2.0**-24 * 2000 * 2 * mass + 1e-6)
    c.q /= 40
    check(c, scale=1e-3)


def test_rising_scores_move_the_maximum():
    c = Cache([(1, 2000), (64, 900)], 2, 2, 64, 16, torch.float32, 5)
    for b, (_, kv) in enumerate(c.lens):
        for p in range(kv):
            c.k[int(c.table[b, p // 16]), :, p % 16] *= 0.02 + 4.0 * p / kv
    check(c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_is_not_seen_does_not_matter(dtype, bad):
    """Everything beyond the lengths, and keys and values that only later queries see, may hold anything."""
    for lens, heads in (([(40, 170), (1, 33), (65, 65)], 4), ([(600, 700)], 64)):
        c = Cache(lens, heads, 2, 64, 16, TYPES[dtype], 6)
        clean_k, clean_v = c.k.clone(), c.v.clone()
        used = torch.zeros(c.k.shape[0], 16, dtype=torch.bool, device="cuda")
        for b, (_, kv) in enumerate(c.lens):
            for p in range(kv):
                used[int(c.table[b, p // 16]), p % 16] = True
        c.k.transpose(1, 2)[~used] = bad
        c.v.transpose(1, 2)[~used] = bad
        check(c)
        check(c, causal=False)
        # a later token's key and value: only queries from it on may notice
        c.k, c.v = clean_k.clone(), clean_v.clone()
        n, kv = c.lens[0]
        p = kv - 7
        pg = int(c.table[0, p // 16])
        c.v[pg, :, p % 16, 3] = bad
        from paper_2604_09975_amd import clear as K
        out = K.ckks_clear_attend(c.q, *c.args())
        want, _, mass = attend_ref(c)
        close(out, want, attend_bound(c, torch.where(torch.isfinite(want), want, 0.0), mass), "value")
        assert torch.isfinite(out[:n - 7]).all() and not torch.isfinite(out[n - 7:n, :, 3]).any()
        c.v = clean_v.clone()
        c.k[pg, :, p % 16] = bad
        out = K.ckks_clear_attend(c.q, *c.args())
        c.k = clean_k
        want, _, mass = attend_ref(c)
        close(out[:n - 7], want[:n - 7], attend_bound(c, want, mass)[:n - 7], "key")
        # before the window
        c.v[int(c.table[0, 0]), :, 0] = bad
        c.k[int(c.table[0, 0]), :, 0] = bad
        out = K.ckks_clear_attend(c.q, *c.args(), window=40)
        c.k, c.v = clean_k, clean_v
        want, _, mass = attend_ref(c, window=40)
        close(out[n - 30:n], want[n - 30:n], attend_bound(c, want, mass)[n - 30:n], "window")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [96, 128, 200])
def test_wide_heads_do_not_meet_what_they_do_not_see(dim, dtype):
    """Chunks large enough for every form of shared tiles, pages that hold whole tiles and pages that do not."""
    from paper_2604_09975_amd import clear as K
    for page in (48, 64):
        c = Cache([(900, 1000), (90, 300)], 64, 4, dim, page, TYPES[dtype], dim + page)
        last = {b: (int(c.table[b, (kv - 1) // page]), (kv - 1) % page) for b, (_, kv) in enumerate(c.lens)}
        for pg, row in last.values():  # beyond the lengths
            c.k[pg, :, row + 1:] = math.nan
            c.v[pg, :, row + 1:] = math.inf
        check(c)
        check(c, window=130)
        n, kv = c.lens[0]
        pg, row = last[0]
        c.k[pg, :, row] = 0.0
        c.v[pg, 1, row, dim - 1] = math.inf  # the last token's: its own query's alone, and the heads' that share it
        out = K.ckks_clear_attend(c.q, *c.args())
        assert torch.isfinite(out[:n - 1]).all() and torch.isfinite(out[n:]).all()
        odd = ~torch.isfinite(out[n - 1])
        assert odd[16:32, dim - 1].all() and int(odd.sum()) == 16


def test_pages_out_of_range_read_as_zeros():
    c = Cache([(3, 70)], 4, 2, 64, 16, torch.float16, 7)
    hole = int(c.table[0, 2])
    c.page_table[0, 2] = -1
    from paper_2604_09975_amd import clear as K
    one = K.ckks_clear_attend(c.q, *c.args())
    c.page_table[0, 2] = c.k.shape[0]
    two = K.ckks_clear_attend(c.q, *c.args())
    c.page_table[0, 2] = hole
    c.k[hole] = 0
    c.v[hole] = 0
    assert torch.equal(one, two) and torch.equal(one, check(c))


def test_a_length_beyond_the_table_is_its_end():
    from paper_2604_09975_amd import clear as K
    c = Cache([(4, 48)], 4, 2, 64, 16, torch.float16, 8)
    want = K.ckks_clear_attend(c.q, *c.args())
    c.kv_len += 1000
    assert torch.equal(want, K.ckks_clear_attend(c.q, *c.args()))


def test_strided_queries_and_outputs():
    from paper_2604_09975_amd import clear as K
    c = Cache([(9, 100), (1, 64)], 6, 3, 64, 16, torch.bfloat16, 9)
    want = check(c)
    room = randn(gen(1), c.total, 6 * 64 + 100, dtype=torch.bfloat16)
    q = room[:, 33:33 + 384].view(c.total, 6, 64)
    q.copy_(c.q)
    out = torch.zeros(6, c.total, 65, dtype=torch.bfloat16, device="cuda")
    K.ckks_clear_attend(q, *c.args(), out=out[:, :, 1:].transpose(0, 1))
    assert torch.equal(out[:, :, 1:].transpose(0, 1), want) and not out[:, :, 0].any()


def test_more_sequences_than_a_wave():
    check(Cache([(1 + i % 3, 1 + i % 3 + (i * 37) % 90) for i in range(150)], 2, 1, 64, 16, torch.float16, 10))


def test_a_cache_beyond_32_bit_offsets():
    from paper_2604_09975_amd import clear as K
    n_pages = 1100000
    k, v = (torch.zeros(n_pages, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2))   # 2.25e9 entries each
    c = Cache([(1, 40), (17, 48)], 4, 2, 64, 16, torch.float16, 12)
    want = check(c)
    far = torch.tensor([[n_pages - 1, n_pages - 5, 17], [n_pages - 9, 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    k[far.flatten().long()], v[far.flatten().long()] = c.k[c.page_table.flatten().long()], c.v[c.page_table.flatten().long()]
    assert torch.equal(want, K.ckks_clear_attend(c.q, k, v, far, c.q_start, c.kv_len))


def test_same_bits_every_time():
    from paper_2604_09975_amd import clear as K
    c = Cache([(1, 9000), (1, 5000)], 8, 2, 128, 64, torch.bfloat16, 13)
    one = K.ckks_clear_attend(c.q, *c.args())
    for _ in range(5):
        assert torch.equal(one, K.ckks_clear_attend(c.q, *c.args()))


def test_no_tokens():
    from paper_2604_09975_amd import clear as K
    c = Cache([(0, 20)], 4, 2, 64, 16, torch.float16, 14)
    assert K.ckks_clear_attend(c.q, *c.args()).shape == (0, 4, 64)


def test_refusals():
    from paper_2604_09975_amd import binding as B
    from paper_2604_09975_amd import clear as K
    c = Cache([(4, 20)], 6, 2, 64, 16, torch.float16, 15)
    with pytest.raises(B.CkksError):
        K.ckks_clear_attend(c.q[:, :5], *c.args())            # 5 heads over 2
    with pytest.raises(B.CkksError):
        K.ckks_clear_attend(c.q, *c.args(), causal=False, window=4)
    for scale in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(B.CkksError):
            K.ckks_clear_attend(c.q, *c.args(), scale=scale)
    with pytest.raises(B.CkksError):
        K.ckks_clear_attend(c.q, *c.args(), out=c.q)
    with pytest.raises(TypeError):
        K.ckks_clear_attend(c.q.float(), *c.args())
    with pytest.raises(ValueError):
        K.ckks_clear_attend(c.q, c.k, c.v[:1], c.page_table, c.q_start, c.kv_len)
    with pytest.raises(ValueError):
        K.ckks_clear_attend(c.q[..., :32], *c.args())
    with pytest.raises(ValueError):
        K.ckks_clear_attend(c.q, *c.args(), lse=torch.empty(4, 5, device="cuda"))
    wide = torch.zeros(2, 2, 16, 264, dtype=torch.float16, device="cuda")
    with pytest.raises(B.CkksError):
        K.ckks_clear_attend(torch.zeros(4, 2, 264, dtype=torch.float16, device="cuda"), wide, wide, c.page_table, c.q_start, c.kv_len)
