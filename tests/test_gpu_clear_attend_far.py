"""Attention at the last positions that a table may reach, just below 2^31."""
import pytest
import torch

from tests.clear_util import TINY, TYPES, U, close, gen, randn

pytestmark = pytest.mark.gpu

PAGE, N_PAGES = 16, 37


@pytest.fixture(scope="module")
def table():
    at = torch.arange((1 << 27) - 1, device="cuda", dtype=torch.int32)
    return torch.remainder(at, N_PAGES, out=at)[None]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,heads,kv_heads,dim", [(1, 2, 1, 8), (1, 4, 2, 128), (40, 2, 1, 64), (900, 32, 2, 64), (900, 32, 2, 128), (300, 16, 2, 256)])
def test_windows_that_end_below_two_to_the_31(table, n, heads, kv_heads, dim, dtype):
    from paper_2604_09975_amd import clear as K
    g, dtype, window = gen(n + dim), TYPES[dtype], 150
    kp, vp = (randn(g, N_PAGES, kv_heads, PAGE, dim, dtype=dtype) for _ in range(2))
    q = randn(g, n, heads, dim, dtype=dtype)
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    for kv in ((1 << 31) - 16, (1 << 31) - 33, (1 << 31) - 64, (1 << 31) - 129):
        lse = torch.empty(n, heads, device="cuda")
        out = K.ckks_clear_attend(q, kp, vp, table, start, torch.tensor([kv], dtype=torch.int32, device="cuda"), window=window, lse=lse)
        p = torch.arange(kv - n - window, kv, device="cuda")                 # all that some query sees, and a little more
        k, v = (x[table[0, p // PAGE].long(), :, p % PAGE].double() for x in (kp, vp))
        t = torch.arange(kv - n, kv, device="cuda")[:, None]
        seen = (p <= t) & (p > t - window)
        for h in range(heads):
            kh, vh = k[:, h * kv_heads // heads], v[:, h * kv_heads // heads]
            s = torch.where(seen, q[:, h].double() @ kh.t().contiguous() * dim**-0.5, -torch.inf)
            w = torch.softmax(s, 1)
            want, mass = w @ vh, w @ vh.abs()
            # the bounds of `attend_bound`
            close(out[:, h], want, U[dtype] * want.abs() + ((0 if dtype is torch.float32 else 2 * U[dtype]) + 2.0**-13) * mass + TINY[dtype], (kv, h))
            wl = torch.logsumexp(s, 1)
            close(lse[:, h], wl, 2.0**-13 * (1 + wl.abs()), (kv, h))
