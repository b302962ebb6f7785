"""The draw of a token where its numbers are smallest: limits below every weight, tokens of very little weight, a million of them."""
import math

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


@pytest.mark.parametrize("vocab", [4000, 50257, 131072, 1 << 20])
def test_a_tail_of_small_weights(vocab):
    """One token that has nearly all of the weight, behind many that have 1e-13 of it each: which of those is drawn, and its probability.
    (The draw's sums are known to 2^-41 of themselves, and a step from one of the tail to the next is 2^-20 of the tail's.)"""
    g = gen(vocab)
    for spread in (0.0, 0.5):
        logits = math.log(1e-13) + spread * randn(g, 1, vocab)
        logits[0, -1] = 0.0
        tail = float(torch.exp(logits[0, :-1].double()).sum())
        us = [0.0, math.nan, tail / 1000, 2.0**-25, 2.0**-24, 0.5, 1 - 2.0**-24, 1.0] + [tail * x for x in (0.1, 0.3, 0.5, 0.7, 0.9)]
        rows = logits.expand(len(us), -1)
        check(rows, us)
        check(rows, us, min_p=[1e-14] * len(us))
        check(rows, us, top_k=[vocab // 3] * len(us))
        check(rows, us, top_k=[200] * len(us))
        check(rows, us, top_k=[3000] * len(us), min_p=[1e-20] * len(us))
        check(rows, us, temperature=[2.0] * len(us))
        some = [0, 1, 3, 4, 5]  # with top_p the last of the tail that is kept, one of many alike, hangs on sums to 2^-43
        check(rows[some], [us[i] for i in some], top_p=[1 - 2.0**-24] * len(some))
        check(rows[some], [us[i] for i in some], top_p=[1 - 2.0**-24] * len(some), top_k=[vocab // 2] * len(some))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [2, 7, 300, 9000, 131072, 1 << 20])
def test_the_first_and_the_last_token_kept_may_weigh_little(vocab, dtype):
    """u of 0 takes the first token kept, u of 1 the last, down to weights of 2^-64; below that a logit counts as -infinity."""
    from paper_2604_09975_amd import clear as K
    logits = torch.full((3, vocab), -math.inf, device="cuda", dtype=TYPES[dtype])
    logits[:, 1] = 0.0
    logits[0, 0], logits[0, -1] = -40.0, -40.0 if vocab > 2 else 0.0
    logits[1, 0], logits[1, -1] = -44.25, -44.25 if vocab > 2 else 0.0
    logits[2, 0], logits[2, -1] = -44.5, -44.5 if vocab > 2 else 0.0
    known = logits.clone()
    known[2, 0] = -math.inf
    if vocab > 2:
        known[2, -1] = -math.inf
    for more in ({}, {"top_k": [3] * 3}, {"top_k": [290] * 3}, {"min_p": [1e-30] * 3}, {"top_k": [290] * 3, "min_p": [1e-25] * 3}):
        for u, at in ((0.0, (0, 0, 1)), (math.nan, (0, 0, 1)), (1.0, (vocab - 1, vocab - 1, 1)), (math.inf, (vocab - 1, vocab - 1, 1)), (1 - 2.0**-24, (1, 1, 1))):
            assert check(known, [u] * 3, **more).tolist() == list(at)
            args = {k: torch.tensor(v, device="cuda", dtype=torch.int32 if k == "top_k" else torch.float32) for k, v in more.items()}
            assert K.ckks_clear_sample(logits, torch.full((3,), u, device="cuda"), **args).tolist() == list(at)



@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_a_mask_leaves_empty_or_with_one_token(dtype):
    """-1 for a row of -infinity or NaN alone, whatever the limits and the temperature; the one token that is left, or that outweighs all."""
    low = torch.finfo(TYPES[dtype]).min
    logits = torch.full((4, 5000), -math.inf, device="cuda", dtype=TYPES[dtype])
    logits[1] = math.nan
    logits[2] = low
    logits[2, 77] = 0.5
    logits[3, 4321] = low
    for u in (0.0, 0.5, 1.0):
        for temperature in (1.0, 0.0, 5.0, math.inf, math.nan):
            for more in ({}, {"top_k": 5}, {"top_k": 900}, {"top_p": 0.6}, {"min_p": 0.2}, {"top_k": 100, "top_p": 0.9}):
                got = check(logits, [u] * 4, temperature=[temperature] * 4, **{k: [x] * 4 for k, x in more.items()}).tolist()
                assert got[:2] == [-1, -1]
                assert got[3] == 4321
                assert got[2] == 77 or temperature == math.inf
