"""Plain forms in 64 bits of the steps in the clear, and the bounds that their tests hold the kernels to.

U is the unit roundoff of a type: a result rounded once is off by U * |result| at most.  What 32-bit sums add is bounded
per test from the number of terms added one after the other and their absolute sum.
"""
import math

import torch

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
TINY = {torch.float32: 2.0**-126, torch.float16: 2.0**-24, torch.bfloat16: 2.0**-126}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def close(got, want, bound, what=""):
    """Elementwise |got - want| <= bound; not-a-number and infinities in the same places."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    odd = ~fine & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd]), what
    off = (got - want).abs()[fine] - bound.expand_as(want)[fine]
    assert off.numel() == 0 or off.max().item() <= 0, (what, off.max().item())


def norm_ref(x, w, b, eps):
    """(y, mean, rstd, xh) in 64 bits."""
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    xh = (x - mean) * rstd
    return xh * (1 if w is None else w.double()) + (0 if b is None else b.double()), mean, rstd, xh


class Cache:
    """A paged cache with its batch: sequences of (new tokens, keys in all); pages in random order."""

    def __init__(self, lens, heads, kv_heads, dim, page, dtype, seed, spare=2, width=None, layout="head"):
        g = gen(seed)
        self.lens, self.heads, self.kv_heads, self.dim, self.page, self.dtype = lens, heads, kv_heads, dim, page, dtype
        need = [max(0, -(-kv // page)) for _, kv in lens]
        n_pages = sum(need) + spare
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))[:sum(need)].tolist()
        self.table = torch.full((len(lens), max(need + [1]) if width is None else width), -1, dtype=torch.int32)
        for b, k in enumerate(need):
            self.table[b, :k] = torch.tensor(order[:k], dtype=torch.int32)
            order = order[k:]
        self.page_table = self.table.cuda()
        starts = [0]
        for n, _ in lens:
            starts.append(starts[-1] + n)
        self.starts, self.total = starts, starts[-1]
        self.q_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device="cuda")
        if layout == "head":  # [page][head][token][dim]
            self.k, self.v = (randn(g, n_pages, kv_heads, page, dim, dtype=dtype) for _ in range(2))
        elif layout == "token":  # [page][token][head][dim]
            self.k, self.v = (randn(g, n_pages, page, kv_heads, dim, dtype=dtype).transpose(1, 2) for _ in range(2))
        else:  # keys and values of a page side by side
            both = randn(g, n_pages, 2, kv_heads, page, dim, dtype=dtype)
            self.k, self.v = both[:, 0], both[:, 1]
        self.q = randn(g, self.total, heads, dim, dtype=dtype)

    def args(self):
        return self.k, self.v, self.page_table, self.q_start, self.kv_len

    def keys(self, b, which):
        """[kv][kv_heads][dim] of sequence b in 64 bits."""
        kv = self.lens[b][1]
        t = self.k if which == "k" else self.v
        pages = self.table[b, :-(-kv // self.page)].long().cuda()
        return t[pages].transpose(1, 2).reshape(-1, self.kv_heads, self.dim)[:kv].double()


def attend_ref(c, causal=True, window=0, scale=None):
    """(out, lse, sum_j p_j |v_j|) of every token and head in 64 bits.  Only what a query sees enters its sums."""
    scale = c.dim**-0.5 if scale is None else scale
    out = torch.zeros(c.total, c.heads, c.dim, dtype=torch.float64, device="cuda")
    mass = torch.zeros_like(out)
    lse = torch.full((c.total, c.heads), -math.inf, dtype=torch.float64, device="cuda")
    group = c.heads // c.kv_heads
    for b, (n, kv) in enumerate(c.lens):
        if not n or kv <= 0:
            continue
        k, v = c.keys(b, "k"), c.keys(b, "v")
        t = torch.arange(kv - n, kv, device="cuda")[:, None]
        j = torch.arange(kv, device="cuda")[None]
        seen = torch.ones(n, kv, dtype=torch.bool, device="cuda")
        if causal:
            seen = j <= t
            if window:
                seen = seen & (j > t - window)
        some = seen.any(1)
        odd = ~torch.isfinite(v)
        for h in range(c.heads):
            kh, vh = k[:, h // group], v[:, h // group]
            s = c.q[c.starts[b]:c.starts[b + 1], h].double() @ kh.t().contiguous() * scale
            s = torch.where(seen, s, -math.inf)
            p = torch.where(some[:, None], torch.softmax(s, 1), 0.0)
            rows = slice(c.starts[b], c.starts[b + 1])
            clean = torch.where(odd[:, h // group], 0.0, vh)
            res = p @ clean
            mass[rows, h] = p @ clean.abs()
            if odd[:, h // group].any():
                for e in torch.nonzero(odd[:, h // group].any(1)).flatten().tolist():
                    add = torch.where(odd[e, h // group], vh[e], 0.0)
                    res = torch.where(seen[:, e:e + 1], res + add, res)
            out[rows, h] = res
            lse[rows, h] = torch.logsumexp(s, 1)
    return out, lse, mass


def attend_bound(c, want, mass, scale=None):
    """Weights rounded to the type (twice U of their sum: numerator and, through it, the quotient), the result rounded once,
    and 2^-13 of the mass for the scores: a 32-bit sum of dim products of size 1 to 10 is off by less, and so is its exponential."""
    u = U[c.dtype]
    weight = 0.0 if c.dtype is torch.float32 else 2 * u
    return u * want.abs() + (weight + 2.0**-13) * mass + TINY[c.dtype]
