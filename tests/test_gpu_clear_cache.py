"""Appending to the paged cache: every entry of the pages afterwards, against the plain form."""
import pytest
import torch

from tests.clear_util import TINY, TYPES, U, Cache, close, gen, randn

pytestmark = pytest.mark.gpu


def tables(n_pos, rot):
    angle = torch.arange(n_pos, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / max(rot, 1))
    return angle.cos().float(), angle.sin().float()


def rotate(x, c, s, interleaved):
    """(rotated, bound) of [n][heads][dim] in 64 bits: two products and a sum in 32 bits, rounded once."""
    u, dtype = U[x.dtype], x.dtype
    x, h = x.double().clone(), c.shape[-1]
    c, s = c.double()[:, None], s.double()[:, None]
    i, j = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    a, b = x[..., i].clone(), x[..., j].clone()
    size = torch.zeros_like(x)
    size[..., i] = size[..., j] = a.abs() + b.abs()
    x[..., i], x[..., j] = a * c - b * s, b * c + a * s
    return x, u * x.abs() * (size > 0) + 3 * 2.0**-24 * size + TINY[dtype] * (size > 0)


def run(c, rot, interleaved, seed, with_q=True, positions=None, in_place=False):
    from paper_2604_09975_amd import clear as K
    g = gen(seed)
    # queries, keys and values as columns of one array
    cols = (c.heads + 2 * c.kv_heads) * c.dim
    qkv = randn(g, c.total, cols, dtype=c.dtype)
    q = qkv[:, :c.heads * c.dim].view(c.total, c.heads, c.dim)
    k = qkv[:, c.heads * c.dim:(c.heads + c.kv_heads) * c.dim].view(c.total, c.kv_heads, c.dim)
    v = qkv[:, (c.heads + c.kv_heads) * c.dim:].view(c.total, c.kv_heads, c.dim)
    n_pos = c.page_table.shape[1] * c.page
    cos, sin = tables(n_pos, rot) if rot else (None, None)
    pos = torch.cat([torch.arange(kv - n, kv) for n, kv in c.lens]).cuda()
    turn = positions if positions is not None else pos
    want_k, want_v = c.k.double(), c.v.double()
    bound = torch.zeros_like(want_k)
    kd, kb = k.double(), torch.zeros(k.shape, dtype=torch.float64, device="cuda")
    qd, qb = q.double().clone(), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    if rot:
        at = turn.long().clamp(0, n_pos - 1)
        kd, kb = rotate(k, cos[at], sin[at], interleaved)
        qd, qb = rotate(q, cos[at], sin[at], interleaved)
        off = (turn < 0) | (turn >= n_pos)
        kd[off, :, :rot] = float("nan")
        qd[off, :, :rot] = float("nan")
    for b, (n, kv) in enumerate(c.lens):
        for i in range(n):
            t, p = c.starts[b] + i, kv - n + i
            if p < 0:
                continue
            pg = int(c.table[b, p // c.page])
            if not 0 <= pg < c.k.shape[0]:
                continue
            want_k[pg, :, p % c.page], want_v[pg, :, p % c.page] = kd[t], v[t].double()
            bound[pg, :, p % c.page] = kb[t]
    v0 = v.clone()
    out = K.ckks_clear_cache_append(k, v, *c.args(), cos=cos, sin=sin, interleaved=interleaved,
                                    positions=positions, q=q if with_q else None, q_out=q if in_place else None)
    close(c.k, want_k, bound, "keys")
    assert torch.equal(c.v.double(), want_v)
    assert torch.equal(v, v0)
    if with_q:
        close(out, qd, qb, "queries")
    else:
        assert out is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,rot,interleaved", [(64, 64, False), (64, 0, False), (128, 64, False), (80, 40, False), (128, 128, True),
                                                 (96, 36, True), (8, 2, True), (8, 2, False), (256, 256, False), (72, 18, False), (16, 6, True)])
def test_pages_after_append(dim, rot, interleaved, dtype):
    lens = [(5, 5), (1, 40), (17, 33), (0, 9), (3, 3)]
    run(Cache(lens, 6, 2, dim, 16, TYPES[dtype], dim + rot), rot, interleaved, rot + 1)


@pytest.mark.parametrize("page", [1, 3, 16, 100, 256])
@pytest.mark.parametrize("layout", ["head", "token", "both"])
def test_page_sizes_and_layouts(page, layout):
    run(Cache([(40, 40), (1, 257), (130, 300)], 4, 4, 32, page, torch.float16, page, layout=layout), 32, False, page)


def test_single_tokens_of_many_sequences():
    """More sequences than the block's copy of their starts holds, and one less."""
    for n in (1, 65, 1024, 1025, 1300):
        run(Cache([(1, 1 + (7 * i) % 50) for i in range(n)], 2, 1, 16, 16, torch.bfloat16, n), 16, False, n)


def test_without_queries_in_place_and_own_positions():
    lens = [(9, 20), (4, 4)]
    run(Cache(lens, 4, 2, 64, 16, torch.bfloat16, 1), 64, False, 1, with_q=False)
    run(Cache(lens, 4, 2, 64, 16, torch.float32, 2), 64, False, 2, in_place=True)
    run(Cache(lens, 4, 2, 64, 16, torch.float32, 2), 32, True, 2, in_place=True)
    places = torch.randint(0, 32, (13,), dtype=torch.int32, device="cuda", generator=gen(3))
    run(Cache(lens, 4, 2, 64, 16, torch.float16, 3), 64, False, 3, positions=places)
    places[3], places[12] = -1, 32          # no such angle
    run(Cache(lens, 4, 2, 64, 16, torch.float16, 4), 32, False, 4, positions=places)


def test_tokens_before_the_cache_and_pages_out_of_range():
    c = Cache([(6, 2), (5, 70), (3, 3)], 2, 2, 32, 16, torch.float32, 5)
    c.table[1, 4], c.table[2, 0] = -1, 1 << 30
    c.page_table = c.table.cuda()
    run(c, 0, False, 5)
    # a length beyond the table is taken as the table's end
    from paper_2604_09975_amd import clear as K
    c = Cache([(4, 32)], 2, 2, 32, 16, torch.float32, 6)
    k = torch.ones(4, 2, 32, device="cuda")
    long = torch.tensor([1000], dtype=torch.int32, device="cuda")
    before = c.k.clone()
    K.ckks_clear_cache_append(k, k, c.k, c.v, c.page_table, c.q_start, long)
    pg = int(c.table[0, 1])
    before[pg, :, 12:] = 1
    assert torch.equal(c.k, before)


def test_a_cache_beyond_32_bit_offsets():
    from paper_2604_09975_amd import clear as K
    n_pages = 2100000
    k = torch.zeros(n_pages, 2, 16, 64, dtype=torch.float16, device="cuda")   # 4.3e9 entries
    v = torch.zeros(1, 2, 16, 64, dtype=torch.float16, device="cuda").expand(n_pages, 2, 16, 64)
    v = torch.zeros_like(k)
    table = torch.tensor([[5, n_pages - 1, n_pages // 2 + 7]], dtype=torch.int32, device="cuda")
    new = randn(gen(1), 40, 2, 64, dtype=torch.float16)
    start, length = torch.tensor([0, 40], dtype=torch.int32, device="cuda"), torch.tensor([40], dtype=torch.int32, device="cuda")
    K.ckks_clear_cache_append(new, -new, k, v, table, start, length)
    for i, pg in enumerate(table[0].tolist()):
        part = new[i * 16:(i + 1) * 16].transpose(0, 1)
        n = part.shape[1]
        assert torch.equal(k[pg, :, :n], part) and torch.equal(v[pg, :, :n], -part)
    assert int((k[:, 0, 0, 0] != 0).sum()) == 3


def test_refusals():
    from paper_2604_09975_amd import binding as B
    from paper_2604_09975_amd import clear as K
    c = Cache([(4, 4)], 4, 2, 64, 16, torch.float16, 7)
    k = randn(gen(2), 4, 2, 64, dtype=torch.float16)
    cos, sin = tables(16, 64)
    with pytest.raises(ValueError):
        K.ckks_clear_cache_append(k[:, :1], k, *c.args())
    with pytest.raises(ValueError):
        K.ckks_clear_cache_append(k[:3], k, *c.args())
    with pytest.raises(TypeError):
        K.ckks_clear_cache_append(k.float(), k, *c.args())
    with pytest.raises(TypeError):
        K.ckks_clear_cache_append(k, k, c.k, c.v, c.page_table.long(), c.q_start, c.kv_len)
    with pytest.raises(ValueError):
        K.ckks_clear_cache_append(k, k, c.k, c.v, c.page_table, c.q_start[:1], c.kv_len)
    with pytest.raises(TypeError):
        K.ckks_clear_cache_append(k, k, *c.args(), cos=cos)
    with pytest.raises(ValueError):
        K.ckks_clear_cache_append(k, k, *c.args(), cos=cos, sin=sin[:4])
    with pytest.raises(B.CkksError):
        K.ckks_clear_cache_append(k, k, *c.args(), cos=torch.cat((cos, cos), 1), sin=torch.cat((sin, sin), 1))   # wider than a head
    with pytest.raises(B.CkksError):
        K.ckks_clear_cache_append(c.k[0].transpose(0, 1)[:4], k, *c.args())   # the pages themselves
    with pytest.raises(ValueError):
        K.ckks_clear_cache_append(k, k, *c.args(), q_out=k)
    odd = Cache([(4, 4)], 4, 2, 64, 16, torch.float16, 7)
    with pytest.raises(B.CkksError):
        K.ckks_clear_cache_append(k[..., :20], k[..., :20], odd.k[..., :20], odd.v[..., :20], odd.page_table, odd.q_start, odd.kv_len)
