"""New tokens into pages of 8 bits and back, against 64 bits: codes and powers to the last bit."""
import math

import pytest
import torch

from tests.clear_util import TINY, TYPES, U, close, gen, randn
from tests.packed_util import FORMATS, PackedCache, pack_ref, powers, same, values

pytestmark = pytest.mark.gpu


def turn_ref(x, cos, sin, interleaved):
    h = cos.shape[-1]
    if not h:
        return x
    c, s, out = cos[:, None], sin[:, None], x.clone()
    one = slice(0, 2 * h, 2) if interleaved else slice(0, h)
    two = slice(1, 2 * h, 2) if interleaved else slice(h, 2 * h)
    out[..., one] = x[..., one] * c - x[..., two] * s
    out[..., two] = x[..., two] * c + x[..., one] * s
    return out


def norm_ref(x, w, eps):
    r = torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + eps)
    return torch.where(torch.isinf(r) & torch.isfinite(x), 0.0, x / r) * w.double()


def places(c):
    """(row, page or -1, row of the page, position) of each new token."""
    got = []
    for b, (n, kv) in enumerate(c.lens):
        kv = min(kv, c.table.shape[1] * c.page)
        for i in range(n):
            pos = kv - n + i
            page = int(c.table[b, pos // c.page]) if pos >= 0 else -1
            got.append((c.starts[b] + i, page if 0 <= page < c.k.shape[0] else -1, pos % c.page, pos))
    return got


def rows_of(c, seed, wide=False):
    g = gen(seed)
    s = {n: randn(g, c.total, h, c.dim) * torch.exp(2 * randn(g, c.total, h, 1)) for n, h in (("k", c.kv_heads), ("v", c.kv_heads), ("q", c.heads))}
    return {n: x.to(c.dtype) for n, x in s.items()}


def angles(n_pos, rot, seed):
    a = torch.rand(n_pos, rot // 2, generator=gen(seed), device="cuda") * 6.283
    return a.cos(), a.sin()


def check(c, s, cos=None, sin=None, interleaved=False, norms=(None, None), eps=1e-6, positions=None, q=True):
    from paper_2604_09975_amd import clear as K
    at = places(c)
    old = [(x.contiguous().view(torch.uint8).clone(), p.clone()) for x, p in zip(c.codes, c.power)]
    out = K.ckks_clear_packed_append(s["k"], s["v"], *c.args(), cos=cos, sin=sin, interleaved=interleaved, positions=positions,
                                     q=s["q"] if q else None, k_norm=norms[0], q_norm=norms[1] if q else None, eps=eps)
    where = torch.tensor([p for _, _, _, p in at] if positions is None else positions.tolist(), device="cuda")
    inside = torch.zeros(len(at), dtype=torch.bool, device="cuda") if cos is None else (where >= 0) & (where < cos.shape[0])
    pick = where.clamp(0, max(0, 0 if cos is None else cos.shape[0] - 1))

    def ref(x, w):
        x = x.double()
        if w is not None:
            x = norm_ref(x, w, eps)
        if cos is not None:
            cs, sn = (torch.where(inside[:, None], t.double()[pick], math.nan) for t in (cos, sin))
            x = turn_ref(x, cs, sn, interleaved)
        return x
    for i, x in enumerate((ref(s["k"], norms[0]), s["v"].double())):
        val, power = pack_ref(x, c.form)
        codes, z = old[i]
        for row, page, r, _ in at:
            if page >= 0:
                z[page, :, r] = power[row]
        assert torch.equal(c.power[i], z), "powers"
        got, want = values(c.codes[i], c.power[i]), values(codes.view(c.form), old[i][1])
        for row, page, r, _ in at:
            if page >= 0:
                want[page, :, r] = val[row]
        assert same(got, want), "values"
    if q:
        want = ref(s["q"], norms[1])
        plain = norms[1] is None and cos is None
        if plain:
            assert same(out, s["q"])
        else:  # one rounding, of what is known to 2^-45
            close(out, want, U[c.dtype] * 1.0001 * want.nan_to_num().abs() + TINY[c.dtype])
    c.refresh()
    return out


LENS = [(1, 1), (1, 77), (5, 5), (0, 40), (37, 101), (20, 290)]


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,rots", [(8, (8, 2)), (24, (0, 10)), (64, (64, 32)), (80, (80, 40)), (128, (128, 36)), (136, (0, 136)), (256, (256, 6))])
def test_norms_and_rotations(dim, rots, dtype, form):
    for i, rot in enumerate(rots):
        c = PackedCache(LENS, 6, 2, dim, 16, TYPES[dtype], dim + rot, FORMATS[form])
        s, g = rows_of(c, dim), gen(dim)
        w = [1 + 0.2 * randn(g, dim) for _ in range(2)]
        cs = angles(300, rot, rot) if rot else (None, None)
        check(c, s, *cs, norms=w)
        check(c, s, *cs, interleaved=True, norms=[x.to(TYPES[dtype]) for x in w])
        check(c, s, *cs)
        check(c, s, *cs, norms=(w[0], None), eps=0.0)
        check(c, s, *cs, norms=(None, w[1]), q=i == 0)


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("page,layout", [(1, "head"), (5, "token"), (16, "both"), (256, "both"), (48, "token")])
def test_page_sizes_and_layouts(page, layout, form):
    c = PackedCache([(20, 333), (1, 50)], 4, 2, 80, page, torch.bfloat16, page, FORMATS[form], layout=layout)
    spare = c.room[..., 0].clone() if layout == "both" else None
    check(c, rows_of(c, 1), *angles(400, 40, 2), norms=(1 + randn(gen(3), 80), None))
    assert spare is None or (torch.equal(c.room[..., 0], spare) and not c.room[..., -2:].any())


@pytest.mark.parametrize("form", FORMATS)
def test_every_border_of_a_code(form):
    """Values at, beside and between the borders of two codes, of a block's largest and of two powers, of every size."""
    form = FORMATS[form]
    top = 448.0 if form is torch.float8_e4m3fn else 127.0
    grid = pack_ref(torch.linspace(0, top, 20000, dtype=torch.float64, device="cuda")[:, None].expand(-1, 2).contiguous(), form)[0][:, 0].unique()
    mid = torch.cat((grid, (grid[1:] + grid[:-1]) / 2)).float()
    x = torch.cat((mid, mid.nextafter(torch.tensor(1e9, device="cuda")), mid.nextafter(torch.tensor(-1e9, device="cuda")).abs()))
    x = x[x <= top]
    rows = -(-x.numel() // 31)
    x = torch.nn.functional.pad(x, (0, rows * 31 - x.numel())).view(rows, 31)
    tops = torch.tensor([top, math.nextafter(top, 0), top / 2, top / 2 * (1 + 2.0**-23), 1.0, top * 0.51], device="cuda")
    s = []
    for e in (-140, -127, -108, -100, -60, -1, 0, 3, 60, 118):
        for t in tops.tolist():
            y = torch.cat((torch.full((rows, 1), t, device="cuda"), x * torch.where(torch.arange(31, device="cuda") % 2 == 0, 1.0, -1.0)), 1)
            s.append((y.double().clamp(-t, t) * math.ldexp(1.0, e)).float())
    s = torch.stack(s).view(-1, 1, 32)
    c = PackedCache([(s.shape[0], s.shape[0])], 1, 1, 32, 64, torch.float32, 3, form)
    check(c, {"k": s, "v": s.flip(0).contiguous(), "q": s})


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan_stay_in_their_block(dtype, form):
    c = PackedCache([(40, 90)], 2, 2, 96, 16, TYPES[dtype], 5, FORMATS[form])
    s = rows_of(c, 6)
    for i, bad in enumerate((math.inf, -math.inf, math.nan)):
        s["k"][i, 0, 3], s["v"][i + 3, 1, 95], s["q"][i + 6, 0, 40] = bad, bad, bad
    check(c, s)
    assert int((c.power[1] == 255).sum()) == 3
    w = 1 + 0.1 * randn(gen(1), 96)
    out = check(c, s, norms=(w, w))
    assert not torch.isfinite(out[6:9, 0]).all() and torch.isfinite(out[9:]).all()
    check(c, s, *angles(100, 96, 7))
    zero = {n: torch.zeros_like(x) for n, x in s.items()}
    check(c, zero, norms=(w, w), eps=1e-6)
    assert (check(c, zero) == 0).all()


def test_positions_of_their_own_and_angles_out_of_range():
    c = PackedCache([(9, 30), (4, 4)], 4, 2, 64, 16, torch.float16, 7)
    s = rows_of(c, 1)
    pos = torch.tensor([0, 5, 59, 60, -1, 7, 2**31 - 1, -2**31, 1, 2, 3, 4, 5], dtype=torch.int32, device="cuda")
    out = check(c, s, *angles(60, 32, 1), positions=pos)
    odd = torch.isnan(out).any(-1).any(-1)
    assert odd.tolist() == [p < 0 or p >= 60 for p in pos.tolist()] and torch.isfinite(out[..., 32:]).all()
    check(c, s, *angles(20, 64, 1))


def test_what_has_no_place_is_not_stored():
    """Positions before the cache, pages out of range, lengths beyond the table, rows in no sequence."""
    from paper_2604_09975_amd import clear as K
    c = PackedCache([(10, 4), (6, 40), (3, 20)], 4, 2, 64, 16, torch.bfloat16, 8)
    c.table[1, 2] = c.page_table[1, 2] = c.k.shape[0]
    c.table[2, 1] = c.page_table[2, 1] = -7
    s = rows_of(c, 2)
    check(c, s, *angles(50, 64, 3), norms=(1 + randn(gen(1), 64), 1 + randn(gen(2), 64)))
    c.kv_len[1] += 10**6  # the table's end
    c.lens[1] = (6, c.table.shape[1] * 16)
    check(c, s)
    more = {n: torch.cat((x, x[:5])) for n, x in s.items()}  # five rows behind the last sequence
    before = [x.contiguous().view(torch.uint8).clone() for x in c.codes]
    q = K.ckks_clear_packed_append(more["k"], more["v"], *c.args(), q=more["q"])
    assert torch.equal(q, more["q"])
    assert all(torch.equal(x.contiguous().view(torch.uint8), y) for x, y in zip(c.codes, before))
    k = torch.full((c.total + 5, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    K.ckks_clear_packed_read(*c.args(), c.total + 5, torch.bfloat16, k_out=k, v_out=v)
    assert (k[-5:] == 7).all() and (v[-5:] == 7).all()
    gone = [row for row, page, _, _ in places(c) if page < 0]
    assert gone and not k[gone].any() and not v[gone].any()


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,page,layout", [(8, 3, "token"), (64, 16, "head"), (80, 16, "both"), (128, 64, "head"), (256, 1, "token")])
def test_read(dim, page, layout, dtype, form):
    from paper_2604_09975_amd import clear as K
    c = PackedCache(LENS, 6, 3, dim, page, TYPES[dtype], dim, FORMATS[form], layout=layout)
    got = K.ckks_clear_packed_read(*c.args(), c.total, TYPES[dtype])
    again = PackedCache(LENS, 6, 3, dim, page, TYPES[dtype], dim, FORMATS[form], layout=layout)
    for x, pages in zip(got, (c.k, c.v)):
        want = torch.zeros(c.total, 3, dim, dtype=torch.float64, device="cuda")
        for row, pg, r, _ in places(c):
            want[row] = pages[pg, :, r]
        assert torch.equal(x.double(), want)  # eight bits by a power of two: every type holds them
    K.ckks_clear_packed_append(*got, *again.args())
    twice = K.ckks_clear_packed_read(*again.args(), c.total, TYPES[dtype])
    assert all(torch.equal(x, y) for x, y in zip(got, twice))
    # rows of wider arrays, side by side
    room = torch.zeros(c.total, 3, 2 * dim + 5, dtype=TYPES[dtype], device="cuda")
    K.ckks_clear_packed_read(*c.args(), c.total, TYPES[dtype], k_out=room[..., 1:1 + dim], v_out=room[..., 3 + dim:3 + 2 * dim])
    assert torch.equal(room[..., 1:1 + dim], got[0]) and torch.equal(room[..., 3 + dim:3 + 2 * dim], got[1])
    assert not room[..., 0].any() and not room[..., 1 + dim:3 + dim].any() and not room[..., 3 + 2 * dim:].any()


@pytest.mark.parametrize("form", FORMATS)
def test_read_of_every_code_and_power(form):
    """Rounded to the type where it ends; powers of 255 and the codes that are no number."""
    from paper_2604_09975_amd import clear as K
    c = PackedCache([(256, 256)], 1, 1, 256, 256, torch.float32, 1, FORMATS[form])
    page = int(c.table[0, 0])
    for codes, power in zip(c.codes, c.power):
        codes.view(torch.uint8)[page, 0] = torch.arange(256, dtype=torch.uint8, device="cuda")
        power[page, 0] = torch.arange(256, dtype=torch.uint8, device="cuda")[:, None]
    c.refresh()
    for dtype in TYPES.values():
        got, _ = K.ckks_clear_packed_read(*c.args(), 256, dtype)
        want = c.k[page, 0].to(torch.float32).to(dtype)
        assert same(got[:, 0], want), dtype


def test_queries_in_place_among_the_columns_of_a_projection():
    from paper_2604_09975_amd import clear as K
    for norm in (None, 1 + 0.1 * randn(gen(9), 64)):
        c, d = (PackedCache([(9, 100), (300, 300)], 4, 2, 64, 16, torch.bfloat16, 9) for _ in range(2))
        qkv = randn(gen(4), c.total, 8 * 64, dtype=torch.bfloat16)
        want = qkv.clone()
        cs = angles(300, 64, 5)

        def parts(x):
            x = x.view(c.total, 8, 64)
            return x[:, :4], x[:, 4:6], x[:, 6:]
        q, k, v = parts(want)
        out = K.ckks_clear_packed_append(k, v, *d.args(), *cs, q=q, k_norm=norm, q_norm=norm)
        q2, k2, v2 = parts(qkv)
        assert K.ckks_clear_packed_append(k2, v2, *c.args(), *cs, q=q2, q_out=q2, k_norm=norm, q_norm=norm) is q2
        assert torch.equal(q2, out) and torch.equal(k2, k) and torch.equal(v2, v)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(c.codes, d.codes))


def test_more_sequences_than_a_wave_and_many_heads():
    c = PackedCache([(i % 3, i % 3 + (i * 37) % 90) for i in range(300)], 5, 1, 64, 16, torch.float16, 10)
    check(c, rows_of(c, 3), *angles(100, 64, 1))
    c = PackedCache([(2, 50)], 70, 35, 40, 16, torch.float32, 2)
    check(c, rows_of(c, 4), *angles(100, 20, 1), norms=(1 + randn(gen(1), 40), 1 + randn(gen(2), 40)))


def test_a_cache_beyond_32_bit_offsets():
    from paper_2604_09975_amd import clear as K
    n_pages = 2200000
    far = [torch.zeros(n_pages, 2, 16, 64, dtype=torch.int8, device="cuda") for _ in range(2)]  # 4.5e9 entries each
    power = [torch.zeros(n_pages, 2, 16, 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = torch.tensor([[n_pages - 1, n_pages - 5, 17], [n_pages - 9, 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    c = PackedCache([(40, 40), (17, 48)], 4, 2, 64, 16, torch.float16, 12, torch.int8)
    s = rows_of(c, 5)
    check(c, s)
    K.ckks_clear_packed_append(s["k"], s["v"], *far, *power, table, c.q_start, c.kv_len)
    got = K.ckks_clear_packed_read(*far, *power, table, c.q_start, c.kv_len, c.total, torch.float16)
    want = K.ckks_clear_packed_read(*c.args(), c.total, torch.float16)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_refusals():
    from paper_2604_09975_amd import binding as B
    from paper_2604_09975_amd import clear as K
    c = PackedCache([(4, 20)], 6, 2, 64, 16, torch.float16, 15)
    s = rows_of(c, 1)
    k, v, q = s["k"], s["v"], s["q"]
    w = torch.ones(64, device="cuda")
    for call, error in ((lambda: K.ckks_clear_packed_append(k[:, :1], v, *c.args()), ValueError),
                        (lambda: K.ckks_clear_packed_append(k.float(), v, *c.args()), TypeError),
                        (lambda: K.ckks_clear_packed_append(k, v, *c.args(), q_norm=w), ValueError),
                        (lambda: K.ckks_clear_packed_append(k, v, *c.args(), k_norm=w[:32]), ValueError),
                        (lambda: K.ckks_clear_packed_append(k, v, *c.args(), k_norm=w.bfloat16()), TypeError),
                        (lambda: K.ckks_clear_packed_append(k, v, *c.args(), q=q, k_norm=w, q_norm=w.half()), TypeError),
                        (lambda: K.ckks_clear_packed_append(k, v, *c.args(), k_norm=w, eps=-1.0), B.CkksError),
                        (lambda: K.ckks_clear_packed_append(k, v, *c.args(), k_norm=w, eps=math.nan), B.CkksError),
                        (lambda: K.ckks_clear_packed_append(k, v, c.codes[0], c.codes[0], *c.args()[2:]), B.CkksError),
                        (lambda: K.ckks_clear_packed_append(k, v, *c.codes, c.power[0][..., :1], *c.args()[3:]), ValueError),
                        (lambda: K.ckks_clear_packed_append(k, v, c.codes[0].view(torch.uint8), *c.args()[1:]), TypeError),
                        (lambda: K.ckks_clear_packed_append(k, v, *c.args(), cos=torch.zeros(9, 33, device="cuda"), sin=torch.zeros(9, 33, device="cuda")), B.CkksError),
                        (lambda: K.ckks_clear_packed_append(k.requires_grad_(), v, *c.args()), ValueError),
                        (lambda: K.ckks_clear_packed_read(*c.args(), 4, torch.float64), TypeError),
                        (lambda: K.ckks_clear_packed_read(*c.args(), 4, torch.float16, k_out=v, v_out=v), B.CkksError)):
        with pytest.raises(error):
            call()
    assert K.ckks_clear_packed_append(v[:0], v[:0], *c.codes, *c.power, c.page_table, torch.zeros_like(c.q_start), c.kv_len) is None
