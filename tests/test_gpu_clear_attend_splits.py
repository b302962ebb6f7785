"""Chunks of few kv heads over long caches: forms whose waves share a tile, with the keys split over blocks, against 64 bits."""
import math

import pytest
import torch

from tests.clear_util import TYPES, Cache, attend_bound, attend_ref, close
from tests.test_gpu_clear_attend import check

pytestmark = pytest.mark.gpu

LENS = [(1300, 7001), (907, 6003), (1, 3)]
FORMS = [(64, "f16"), (64, "bf16"), (104, "f16"), (128, "f16"), (128, "bf16"), (200, "f16"), (256, "bf16"), (104, "f32"), (128, "f32"), (256, "f32")]


def splits(c, causal=True, window=0):
    """The number of blocks that the workspace says the keys of a row are dealt out to."""
    from paper_2604_09975_amd import clear as K
    args = K._ATTEND(*K._cache(*c.args(), c.total, torch.cuda.current_device()), c.q.data_ptr(), 0, 0, 0, 0, 0, 0, 0, 0, c.heads, window, int(causal), 1.0)
    return K._attend_work(args) // (4 * c.total * c.heads * (c.dim + 1))


@pytest.mark.parametrize("dim,dtype", FORMS)
@pytest.mark.parametrize("page", [48, 64])
def test_shared_tiles_with_split_keys(page, dim, dtype):
    c = Cache(LENS, 8, 2, dim, page, TYPES[dtype], dim + page)
    for how in (dict(), dict(causal=False), dict(window=3500), dict(window=6000)):
        assert splits(c, **how) > 1
        check(c, **how)


@pytest.mark.parametrize("dim,dtype", FORMS)
def test_values_left_out_with_split_keys(dim, dtype):
    """An infinite value that a chunk's last queries alone see, one that a window leaves behind, one that all see."""
    from paper_2604_09975_amd import clear as K
    c = Cache(LENS, 8, 2, dim, 64, TYPES[dtype], dim)
    n, kv = LENS[0]
    for p, h, e, x in ((kv - 7, 1, 3, math.inf), (kv - 800, 0, dim - 1, -math.inf), (2600, 1, 9, math.inf), (50, 0, 5, math.nan)):
        c.v[int(c.table[0, p // 64]), h, p % 64, e] = x
    for how in (dict(), dict(window=4000)):
        assert splits(c, **how) > 1
        out = K.ckks_clear_attend(c.q, *c.args(), **how)
        want, _, mass = attend_ref(c, **how)
        close(out, want, attend_bound(c, torch.where(torch.isfinite(want), want, 0.0), mass), "out")
        assert not torch.isfinite(out[n - 7:n, 4:, 3]).any() and torch.isfinite(out[:n - 7, :, 3]).all() and torch.isfinite(out[n:]).all()
