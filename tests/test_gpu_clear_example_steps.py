"""The example's key holder: what it does with the rows that came back, in 64 bits from those very rows, and the end of its cache."""
import math

import numpy as np
import pytest
import torch

from tests.clear_util import norm_ref

pytestmark = pytest.mark.gpu


def test_logits_of_the_rows_that_came_back():
    """The bounds of the layer norm's tests, through a 32-bit product of 64 terms and the rules (six roundings)."""
    from examples import encrypted_block as X
    block = X.Block(seed=6, max_tokens=64)
    prompt = np.random.default_rng(7).integers(0, X.VOCAB, 21).tolist()
    allowed = set(range(1, X.VOCAB, 2))
    tokens, rows, steps = block.generate(prompt, 9, allowed)
    (w, b), head = block.norms[1], block.head.double()
    y, _, rstd, xh = norm_ref(rows, w, b, 1e-5)
    rho = 1 + rows.double().abs().amax(-1, keepdim=True) * rstd
    off = 2.0**-24 * y.abs() + 2.0**-18 * (w.double().abs() * (1 + xh.abs()) * rho + b.double().abs())
    logits = y @ head
    bound = off @ head.abs() + 66 * 2.0**-24 * (y.abs() @ head.abs())
    for i, got in enumerate(steps):
        t = len(prompt) - 1 + i
        l, e, past = logits[t].clone(), bound[t].clone(), tokens[:t + 1]
        for v in set(past):
            l[v] = l[v] / 1.3 if l[v] > 0 else l[v] * 1.3
            e[v] *= 1.3
        e += 2.0**-21 * (l.abs() + 2.5)
        for v in set(past[len(prompt):]):
            l[v] -= 0.5
        l[7] += 2.0
        hidden = torch.tensor([v not in allowed for v in range(X.VOCAB)], device="cuda")
        assert torch.equal(got == -math.inf, hidden)
        assert ((got.double() - l).abs() <= e)[~hidden].all()
        assert tokens[t + 1] == int(got.argmax())


def test_more_tokens_than_the_cache_holds_are_an_error():
    """A length beyond the table is its end to the calls below: without the check the last tokens would write over one another."""
    from examples import encrypted_block as X
    block = X.Block(seed=8, max_tokens=24)
    prompt = np.random.default_rng(9).integers(0, X.VOCAB, 20).tolist()
    tokens, rows, _ = block.generate(prompt, 5)      # the fifth is not taken in
    assert len(tokens) == 25 and rows.shape[0] == 24
    with pytest.raises(ValueError, match="25 tokens in a cache of 24"):
        block.generate(tokens[-1:], 1)
    assert block.length == 24
