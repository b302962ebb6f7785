"""Queries rotated in place between the new keys and values that they come with, in every order of one array."""
import pytest
import torch

from tests.clear_util import Cache, gen, randn
from tests.test_gpu_clear_cache import tables

pytestmark = pytest.mark.gpu

T, H, D = 13, 4, 64


def parts(order, t, g):
    """(q, k, v) of [t][H][D] as views of one array."""
    if order == "columns":               # [t][3][H][D]
        x = randn(g, t, 3, H, D, dtype=torch.float16)
        return x[:, 0], x[:, 1], x[:, 2]
    if order == "heads":                 # [t][H][3][D]
        x = randn(g, t, H, 3, D, dtype=torch.float16)
        return x[:, :, 0], x[:, :, 1], x[:, :, 2]
    if order == "tokens":                # [t][3 D] for each head, heads outermost
        x = randn(g, H, t, 3, D, dtype=torch.float16).transpose(0, 1)
        return x[:, :, 0], x[:, :, 1], x[:, :, 2]
    x = randn(g, 3, t, H, D, dtype=torch.float16)
    return x[0], x[1], x[2]


@pytest.mark.parametrize("order", ["columns", "heads", "tokens", "apart"])
@pytest.mark.parametrize("t", [1, T])
def test_in_place_between_keys_and_values(t, order):
    from paper_2604_09975_amd import clear as K
    cos, sin = tables(32, D)
    a, b = (Cache([(t, t + 9)], H, H, D, 16, torch.float16, 3) for _ in range(2))
    q, k, v = parts(order, t, gen(4))
    want = K.ckks_clear_cache_append(k.contiguous(), v.contiguous(), *a.args(), cos=cos, sin=sin, q=q.contiguous())
    kept = k.clone(), v.clone()
    out = K.ckks_clear_cache_append(k, v, *b.args(), cos=cos, sin=sin, q=q, q_out=q)
    assert out is q and torch.equal(q, want) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
    assert torch.equal(k, kept[0]) and torch.equal(v, kept[1])


def test_in_place_over_shared_entries_is_refused():
    from paper_2604_09975_amd import binding as B
    from paper_2604_09975_amd import clear as K
    c = Cache([(T, T)], H, H, D, 16, torch.float16, 5)
    x = randn(gen(6), T, 2 * H, D, dtype=torch.float16)
    for q, k, v in ((x[:, :H], x[:, :H], x[:, H:]), (x[:, :H], x[:, H:], x[:, :H]), (x[:, :H], x[:, 1:H + 1], x[:, H:]), (x[:, ::2], x[:, 2:6], x[:, 1::2])):
        with pytest.raises(B.CkksError, match="overlaps"):
            K.ckks_clear_cache_append(k, v, *c.args(), q=q, q_out=q)
