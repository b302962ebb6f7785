"""Plain forms in 64 bits of a cache of 8 bits: the values of codes, the rounding to them, pages and batches."""
import math

import torch

from tests.clear_util import Cache, gen

FORMATS = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
LARGEST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
BLOCK = 32


def code_values(form):
    """The value of each of the 256 codes, in 64 bits."""
    got = []
    for c in range(256):
        if form is torch.int8:
            got.append(float(c if c < 128 else c - 256))
            continue
        e, m = c >> 3 & 15, c & 7
        x = math.nan if c & 127 == 127 else math.ldexp(1 + m / 8, e - 7) if e else math.ldexp(m, -9)
        got.append(-x if c & 128 else x)
    return torch.tensor(got, dtype=torch.float64)


def powers(power):
    """2^(power - 127) in 64 bits, not a number for 255."""
    table = torch.tensor([math.ldexp(1.0, p - 127) for p in range(255)] + [math.nan], dtype=torch.float64, device=power.device)
    return table[power.long()]


def values(codes, power):
    """What codes [..., dim] with power [..., blocks] stand for, in 64 bits."""
    x = code_values(codes.dtype).to(codes.device)[codes.contiguous().view(torch.uint8).long()]
    return x * powers(power).repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]


def pack_ref(x, form):
    """(values of the codes, powers) of 64-bit x [..., dim]: the nearest of a code's values, of two the one whose last bit is 0."""
    grid = code_values(form)[:127 if form is torch.float8_e4m3fn else 128].to(x.device)  # without a sign, rising
    middle = (grid[1:] + grid[:-1]) / 2
    dim, blocks = x.shape[-1], -(-x.shape[-1] // BLOCK)
    out, power = torch.empty_like(x), torch.empty(x.shape[:-1] + (blocks,), dtype=torch.uint8, device=x.device)
    steps = torch.tensor([math.ldexp(LARGEST[form], e) for e in range(-100, 129)], dtype=torch.float64, device=x.device)
    for b in range(blocks):
        y = x[..., b * BLOCK:(b + 1) * BLOCK]
        top = y.abs().amax(-1)
        bad = ~(top < 2.0**128)
        top = torch.where(bad, 0.0, top)
        e = (top[..., None] > steps).sum(-1) - 100
        scale = powers((e + 127).to(torch.uint8))[..., None]
        size = torch.where(bad[..., None], 0.0, y.abs()) / scale
        at = torch.searchsorted(middle, size.contiguous())
        tie = (at < len(middle)) & (middle[at.clamp(max=len(middle) - 1)] == size) & (at % 2 == 1)
        z = torch.copysign(grid[at + tie.long()] * scale, y)
        out[..., b * BLOCK:b * BLOCK + y.shape[-1]] = torch.where(bad[..., None], math.nan, z)
        power[..., b] = torch.where(bad, 255, e + 127).to(torch.uint8)
    return out, power


def same(got, want):
    return torch.equal(got.nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0)) and torch.equal(torch.isnan(got), torch.isnan(want))


class PackedCache(Cache):
    """Pages of random codes of about the size 1, and their values as `k` and `v`, which attend_ref reads."""

    def __init__(self, lens, heads, kv_heads, dim, page, dtype, seed, form=torch.float8_e4m3fn, layout="head", **more):
        super().__init__(lens, heads, kv_heads, dim, page, dtype, seed, **more)
        g, n, blocks = gen(seed + 1000), self.k.shape[0], -(-dim // BLOCK)
        top, unit = LARGEST[form] / 2.5, int(math.log2(LARGEST[form] / 5))

        def codes(*shape):
            x = (torch.randn(*shape, generator=g, device="cuda") * (top / 2)).clamp_(-2 * top, 2 * top)
            return (x.round_() if form is torch.int8 else x).to(form)

        def scale(*shape):
            return (torch.randint(-1, 2, shape, generator=g, device="cuda") + 127 - unit).to(torch.uint8)
        self.form = form
        if layout == "head":
            self.codes = [codes(n, kv_heads, page, dim) for _ in range(2)]
            self.power = [scale(n, kv_heads, page, blocks) for _ in range(2)]
        elif layout == "token":
            self.codes = [codes(n, page, kv_heads, dim).transpose(1, 2) for _ in range(2)]
            self.power = [scale(n, page, kv_heads, blocks).transpose(1, 2) for _ in range(2)]
        else:  # keys, values and their powers side by side in rows of one array, at an odd place
            room = torch.zeros(n, kv_heads, page, 2 * (dim + blocks) + 3, dtype=torch.uint8, device="cuda")
            at = 1
            self.codes, self.power = [], []
            for _ in range(2):
                room[..., at:at + dim] = codes(n, kv_heads, page, dim).view(torch.uint8)
                self.codes.append(room[..., at:at + dim].view(form))
                at += dim
                room[..., at:at + blocks] = scale(n, kv_heads, page, blocks)
                self.power.append(room[..., at:at + blocks])
                at += blocks
            self.room = room
        self.refresh()

    def refresh(self):
        self.k, self.v = (values(c, p) for c, p in zip(self.codes, self.power))

    def args(self):
        return (*self.codes, *self.power, self.page_table, self.q_start, self.kv_len)
