"""The draw of a token where its numbers are smallest: limits below every weight."""
import pytest
import torch

from tests.clear_util import TYPES, gen, randn
from tests.test_gpu_clear_sample import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [3000, 20000])
def test_a_min_p_below_every_weight_takes_nothing_from_the_other_limits(vocab, dtype):
    """Of every size down to the smallest subnormal: each token reaches it, and top_p and top_k hold as they do without it."""
    g = gen(vocab)
    least = [1e-45, 1e-40, 1.17e-38, 1.18e-38, 1e-30, 2.0**-65, 2.0**-64, 2.0**-63, 1e-10]
    logits = (2 * randn(g, len(least), vocab)).to(TYPES[dtype])
    for top_p, top_k in ((0.5, None), (0.9, None), (None, 300), (None, 1000), (0.9, 1000), (0.9, 50), (None, None)):
        limits = {n: [x] * len(least) for n, x in (("top_p", top_p), ("top_k", top_k)) if x is not None}
        # close to 1 and 0: a token outside the limits would be drawn
        for u in (torch.full((len(least),), 1 - 2.0**-24), torch.zeros(len(least)), torch.rand(len(least), generator=torch.Generator().manual_seed(vocab))):
            with_it, without = check(logits, u, min_p=least, **limits), check(logits, u, **limits)
            assert torch.equal(with_it, without)
