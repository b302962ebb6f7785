"""More tokens and rows than one launch has threads for: each row as it comes out of a call of fewer."""
import pytest
import torch

from tests.clear_util import gen, randn

pytestmark = pytest.mark.gpu


def test_tokens():
    from paper_2604_09975_amd import clear as K
    n, page, dim = (1 << 26) + 1000, 1 << 16, 8
    pages = -(-n // page)
    g = gen(1)
    k, v, q = (randn(g, n, 1, dim, dtype=torch.bfloat16) for _ in range(3))
    cos, sin = (randn(g, 1, 1).expand(n, 2).contiguous() for _ in range(2))
    table = torch.arange(pages, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()

    def empty():
        return ([torch.zeros(pages, 1, page, dim, dtype=torch.int8, device="cuda") for _ in range(2)] +
                [torch.zeros(pages, 1, page, 1, dtype=torch.uint8, device="cuda") for _ in range(2)])

    def batch(rows, kv):
        return table, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.tensor([kv], dtype=torch.int32, device="cuda")
    one, two = empty(), empty()
    out = K.ckks_clear_packed_append(k, v, *one, *batch(n, n), cos=cos, sin=sin, q=q)
    step = 1 << 24
    for at in range(0, n, step):
        end = min(at + step, n)
        part = K.ckks_clear_packed_append(k[at:end], v[at:end], *two, *batch(end - at, end), cos=cos, sin=sin, q=q[at:end])
        assert torch.equal(part, out[at:end])
    assert all(torch.equal(a, b) for a, b in zip(one, two)) and all(bool(x.any()) for x in one)
    del out, part, two, q, cos, sin
    got = K.ckks_clear_packed_read(*one, *batch(n, n), n, torch.bfloat16)
    for at in range(0, n, step):
        end = min(at + step, n)
        part = K.ckks_clear_packed_read(*one, *batch(end - at, end), end - at, torch.bfloat16)
        assert all(torch.equal(a, b[at:end]) for a, b in zip(part, got))


@pytest.mark.parametrize("rows,vocab", [((1 << 24) + 77, 8), ((1 << 22) + 5, 9000)])
def test_rows_of_logits(rows, vocab):
    """(The larger vocabulary: the same few rows again and again.)"""
    from paper_2604_09975_amd import clear as K
    g = gen(2)
    u = torch.rand(rows, generator=g, device="cuda")
    if vocab == 8:
        logits = randn(g, rows, vocab, dtype=torch.bfloat16)
    else:
        logits = randn(g, 1, vocab, dtype=torch.bfloat16).expand(rows, -1)
    prob, few = torch.full((rows,), 7.0, device="cuda"), torch.empty(1000, device="cuda")
    got = K.ckks_clear_sample(logits, u, out=torch.full((rows,), -9, dtype=torch.int32, device="cuda"), prob=prob)
    assert int(got.min()) >= 0 and float(prob.max()) <= 1
    for at in (0, (1 << 21) - 500, 1 << 21, (1 << 22) - 995, rows - 1000):
        part = K.ckks_clear_sample(logits[at:at + 1000], u[at:at + 1000], prob=few)
        assert torch.equal(part, got[at:at + 1000]) and torch.equal(few, prob[at:at + 1000])
