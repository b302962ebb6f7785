"""The example with a cache of 8 bits and drawn tokens: each token is the one that the draw's definition gives for the step's logits, and
the cache holds the rows that were appended."""
import numpy as np
import pytest
import torch

from tests.packed_util import values
from tests.test_gpu_clear_sample import draw_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", [torch.int8, torch.float8_e4m3fn])
def test_drawn_tokens(form):
    from examples import encrypted_block as X
    block = X.Block(seed=4, max_tokens=48, packed=form)
    prompt = np.random.default_rng(5).integers(0, X.VOCAB, 21).tolist()
    allowed = set(range(0, X.VOCAB, 3)) | {7}
    draw = np.random.default_rng(6).random(5)
    tokens, rows, steps = block.generate(prompt, 5, allowed, draw)
    assert len(tokens) == 26 and rows.shape == (25, X.WIDTH) and torch.isfinite(rows).all() and block.length == 25
    for i, l in enumerate(steps):
        u = float(np.float32(draw[i]))
        assert tokens[21 + i] == draw_ref(l.double().cpu().numpy(), u, top_k=20, top_p=float(np.float32(0.9)))[0] in allowed
    for codes, power in zip(block.cache[:2], block.cache[2:]):
        got = values(codes, power)
        pages = block.page_table[0].long()
        held = got[pages].transpose(1, 2).reshape(-1, X.KV_HEADS, X.DIM)
        assert held[:25].abs().amax((1, 2)).min() > 0.1 and not held[25:].any()
    with pytest.raises(ValueError):
        block.chunk([1] * 40)
