"""The draw of a token against the definition in 64 bits (sums in 80): the very token, and its probability."""
import math

import numpy as np
import pytest
import torch

from tests.clear_util import TYPES, gen, randn

pytestmark = pytest.mark.gpu


def draw_ref(l, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probability) of one row."""
    l = np.array(l, dtype=np.float64)
    l[np.isnan(l)] = -math.inf
    top = l.max()
    if top == -math.inf:
        return -1, 0.0
    if top == math.inf:
        l = np.where(l == math.inf, 0.0, -math.inf)
        top = 0.0
    if temperature <= 0:
        return int(l.argmax()), 1.0
    t = 1.0 if math.isnan(temperature) else float(temperature)
    with np.errstate(invalid="ignore"):
        w = np.where(l == -math.inf, 0.0, np.exp((l - top) / t)).astype(np.longdouble)
    order = np.argsort(-l, kind="stable")
    order = order[w[order] > 0]
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        before = np.cumsum(w[order]) - w[order]
        n = max(1, int((before < np.longdouble(top_p) * w[order].sum()).sum()))
        order = order[:n]
    if min_p > 0:
        order = order[w[order] >= min(float(min_p), 1.0)]
    order = np.sort(order)
    upto = np.cumsum(w[order])
    u = 0.0 if math.isnan(u) else max(float(u), 0.0)
    at = min(int((upto <= np.longdouble(u) * upto[-1]).sum()), len(order) - 1)
    return int(order[at]), float(w[order[at]] / upto[-1])


NAMES = ("temperature", "top_k", "top_p", "min_p")


def check(logits, u, **more):
    from paper_2604_09975_amd import clear as K
    rows = logits.shape[0]
    prob = torch.full((rows,), 7.0, device="cuda")
    args = {k: torch.tensor(v, device="cuda", dtype=torch.int32 if k == "top_k" else torch.float32) for k, v in more.items()}
    u = torch.as_tensor(u, dtype=torch.float32).cuda()
    kept = logits.clone()
    got = K.ckks_clear_sample(logits, u, **args, prob=prob)
    assert got.dtype is torch.int32 and torch.equal(logits.nan_to_num(nan=3.0), kept.nan_to_num(nan=3.0))
    host, uh = logits.double().cpu().numpy(), u.double().cpu().tolist()
    want = [draw_ref(host[r], uh[r], **{k: args[k][r].item() for k in args}) for r in range(rows)]
    assert got.tolist() == [t for t, _ in want]
    # w and the sum are known to 2^-40, the quotient is rounded once
    assert np.allclose(prob.cpu().numpy(), [p for _, p in want], rtol=2.0**-23, atol=0)
    return got


def settings(rows, seed, vocab):
    r = np.random.default_rng(seed)
    pick = lambda *v: [v[int(r.integers(len(v)))] for _ in range(rows)]  # noqa: E731
    return {"temperature": pick(1.0, 0.7, 1.3, 0.2, 3.0, 0.0), "top_k": pick(0, 1, 2, 5, 50, 1000, vocab, vocab + 7, -3),
            "top_p": pick(1.0, 0.9, 0.5, 0.99, 0.01, 0.0, 1.5, -1.0), "min_p": pick(0.0, 0.1, 0.01, 1.0, 2.0, -1.0)}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 5, 63, 1000, 4096, 8191, 8193, 50257, 131072])
def test_every_limit_beside_every_other(vocab, dtype):
    rows = 24 if vocab < 50000 else 12
    g = gen(vocab)
    logits = (3 * randn(g, rows, vocab)).to(TYPES[dtype])
    u = torch.rand(rows, generator=g, device="cuda")
    check(logits, u)
    check(logits, u, **settings(rows, vocab, vocab))
    s = settings(rows, vocab + 1, vocab)
    for names in (("top_k",), ("top_p",), ("min_p",), ("temperature",), ("top_k", "top_p"), ("top_p", "min_p"), ("top_k", "min_p", "temperature")):
        check(logits, u, **{k: s[k] for k in names})


@pytest.mark.parametrize("vocab", [200001, 1 << 20])
def test_large_vocabularies(vocab):
    g = gen(2)
    for dtype in (torch.float32, torch.bfloat16):
        logits = (2.5 * randn(g, 3, vocab)).to(dtype)
        u = torch.rand(3, generator=g, device="cuda")
        check(logits, u)
        check(logits, u, top_p=[0.9, 0.99, 0.5], top_k=[0, 5000, 70000])
        check(logits, u, min_p=[0.001, 0.1, 0.0], temperature=[0.8, 1.5, 10.0])


@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows(dtype):
    g = gen(3)
    logits = (2.5 * randn(g, 600, 3001)).to(TYPES[dtype])
    check(logits, torch.rand(600, generator=g, device="cuda"), **settings(600, 4, 3001))


def test_every_border_of_u():
    """u at 0, right before 1, at 1 and beyond, below 0 and not a number; and at the borders of four equal tokens."""
    logits = torch.zeros(1, 40, device="cuda").fill_(-math.inf)
    logits[0, [3, 11, 12, 39]] = 2.0
    us = [0.0, 1 - 2.0**-24, 1.0, 7.0, math.inf, -1.0, -math.inf, math.nan, 0.25, 0.5, 0.75, 0.25 - 2.0**-26, 0.5 - 2.0**-25, 0.75 - 2.0**-24]
    got = check(logits.expand(len(us), 40), us)
    assert got.tolist() == [3, 39, 39, 39, 39, 3, 3, 3, 11, 12, 39, 3, 11, 12]


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_logits(dtype):
    """The lowest ids of equal ones, where a limit falls between them: few, more than a list holds, all."""
    for vocab in (7, 300, 5000, 70000):
        for value in (0.0, -3.0, 1e4):
            logits = torch.full((6, vocab), value, device="cuda", dtype=TYPES[dtype])
            u = [0.0, 0.3, 0.5, 0.7, 0.999, 0.1]
            check(logits, u)
            check(logits, u, top_k=[1, 2, vocab // 2, vocab - 1, vocab, 5])
            check(logits, u, top_p=[0.5, 0.25, 0.75, 0.125, 0.999, 0.0])
            check(logits, u, top_k=[4, 4, 4, 4, 4, 4], top_p=[0.5, 0.25, 0.75, 0.74, 0.76, 1.0])
    # two values, and ties on either side of the border
    logits = torch.zeros(8, 3000, device="cuda", dtype=TYPES[dtype])
    logits[:, ::3] = 1.0
    logits[:, 1::100] = 2.0
    check(logits, torch.rand(8, generator=gen(1), device="cuda"), top_k=[29, 30, 31, 500, 1030, 1031, 2999, 3], top_p=[1.0, 0.9, 0.5, 0.3, 0.99, 0.7, 0.98, 0.5])


def test_values_that_lie_close_together():
    """More tokens in a bin than a list holds, all different: the bin is divided again, and again."""
    g = gen(5)
    for spread in (1e-2, 1e-4, 1e-6):
        logits = 5 + spread * torch.rand(6, 60000, generator=g, device="cuda")
        u = torch.rand(6, generator=g, device="cuda")
        check(logits, u, top_k=[1, 100, 1000, 30000, 59999, 0], top_p=[1.0, 0.9, 0.37, 0.5, 1.0, 0.999])
    logits = torch.cat((5 + 1e-3 * torch.rand(4, 30000, generator=g, device="cuda"), -torch.rand(4, 30000, generator=g, device="cuda") * 1e-30), 1)
    check(logits, torch.rand(4, generator=g, device="cuda"), top_k=[30000, 30001, 45000, 29999], temperature=[1.0, 4.0, 100.0, 0.01])


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_nan_and_rows_that_a_mask_leaves_empty(dtype):
    g = gen(6)
    low = torch.finfo(TYPES[dtype]).min
    logits = (2 * randn(g, 8, 5000)).to(TYPES[dtype])
    logits[0] = -math.inf
    logits[1] = math.nan
    logits[2, ::2] = -math.inf
    logits[3, [5, 700, 4999]] = math.inf
    logits[4, 1::2] = math.nan
    logits[5] = low                # the type's lowest value is no mask
    logits[6] = low
    logits[6, 77] = 0.5
    logits[7, :] = -math.inf
    logits[7, 4321] = low
    u = torch.rand(8, generator=g, device="cuda")
    for more in ({}, dict(top_k=[5] * 8), dict(top_p=[0.6] * 8), dict(min_p=[0.2] * 8), dict(temperature=[0.0] * 8), dict(temperature=[math.inf] * 8, top_k=[100] * 8, top_p=[0.9] * 8)):
        got = check(logits, u, **more)
        assert got[:2].tolist() == [-1, -1] and got[6] == 77 or "temperature" in more and got[7] == 4321


@pytest.mark.parametrize("dtype", TYPES)
def test_temperatures_of_every_size(dtype):
    g = gen(7)
    t = [1e-45, 1e-30, 1e-6, 1e-2, 0.3, 30.0, 1e6, 3e38, math.inf, math.nan, -1.0, -math.inf, 0.0, -0.0]
    logits = (3 * randn(g, len(t), 3000)).to(TYPES[dtype])
    u = torch.rand(len(t), generator=g, device="cuda")
    check(logits, u, temperature=t)
    check(logits, u, temperature=t, top_k=[40] * len(t), top_p=[0.8] * len(t))


def test_min_p_beside_limits_that_it_keeps_to_and_that_it_does_not():
    """top_k and top_p around the number and the sum of the tokens that reach min_p; top_p of the top_k's sum."""
    g = gen(11)
    logits = 2 * randn(g, 1, 20000)
    w = torch.exp(logits[0].double() - logits.max().double()).sort(descending=True).values
    n = int((w >= 0.05).sum())
    share = float(w[:n].sum() / w.sum())
    rows = [(k, p) for k in (0, 300, n - 1, n, n + 1, 2 * n, 5000) for p in (1.0, share * 0.9, share * 0.999, share * 1.001, share * 1.2, 0.9)]
    u = torch.rand(len(rows), generator=g, device="cuda")
    check(logits.expand(len(rows), -1), u, top_k=[k for k, _ in rows], top_p=[min(p, 1.0) for _, p in rows], min_p=[0.05] * len(rows))
    check(logits.expand(len(rows), -1).half(), u, top_k=[k for k, _ in rows], top_p=[min(p, 1.0) for _, p in rows], min_p=[0.05] * len(rows), temperature=[0.7] * len(rows))


def test_limits_that_are_not_a_number_are_none():
    g = gen(8)
    logits, u = randn(g, 4, 900), torch.rand(4, generator=g, device="cuda")
    want = check(logits, u)
    nan = torch.full((4,), math.nan, device="cuda")
    from paper_2604_09975_amd import clear as K
    assert torch.equal(want, K.ckks_clear_sample(logits, u, top_p=nan, min_p=nan))


def test_rows_of_a_wider_array_and_given_outputs():
    from paper_2604_09975_amd import clear as K
    g = gen(9)
    for dtype in TYPES.values():
        room = (3 * randn(g, 5, 9001)).to(dtype)
        u, k = torch.rand(5, generator=g, device="cuda"), torch.full((5,), 30, dtype=torch.int32, device="cuda")
        view = room[:, 7:8008]
        want = K.ckks_clear_sample(view.contiguous(), u, top_k=k)
        out = torch.zeros(7, dtype=torch.int32, device="cuda")
        assert K.ckks_clear_sample(view, u, top_k=k, out=out[1:6]).data_ptr() == out[1:].data_ptr()
        assert torch.equal(out[1:6], want) and not out[0] and not out[6]
        one = K.ckks_clear_sample(view[:1].expand(5, -1), u, top_k=k)   # the same row for several numbers
        assert torch.equal(one, K.ckks_clear_sample(view[:1].repeat(5, 1), u, top_k=k))


def test_same_token_every_time():
    from paper_2604_09975_amd import clear as K
    g = gen(10)
    logits, u = (2.5 * randn(g, 64, 50257)).half(), torch.rand(64, generator=g, device="cuda")
    p = torch.full((64,), 0.95, device="cuda")
    prob = torch.empty(64, device="cuda")
    want = K.ckks_clear_sample(logits, u, top_p=p, prob=prob)
    for _ in range(5):
        again = torch.empty(64, device="cuda")
        assert torch.equal(want, K.ckks_clear_sample(logits, u, top_p=p, prob=again)) and torch.equal(prob, again)


def test_refusals():
    from paper_2604_09975_amd import binding as B
    from paper_2604_09975_amd import clear as K
    x, u = torch.zeros(3, 50, device="cuda"), torch.zeros(3, device="cuda")
    for call, error in ((lambda: K.ckks_clear_sample(x[0], u[:1]), ValueError), (lambda: K.ckks_clear_sample(x, u[:2]), ValueError),
                        (lambda: K.ckks_clear_sample(x, u.double()), TypeError), (lambda: K.ckks_clear_sample(x, u, top_k=u), TypeError),
                        (lambda: K.ckks_clear_sample(x.double(), u), TypeError), (lambda: K.ckks_clear_sample(x[:, :0], u), B.CkksError),
                        (lambda: K.ckks_clear_sample(x.t().contiguous().t(), u), ValueError),
                        (lambda: K.ckks_clear_sample(torch.zeros(1, (1 << 20) + 1, device="cuda"), u[:1]), B.CkksError),
                        (lambda: K.ckks_clear_sample(x, u, prob=u), B.CkksError), (lambda: K.ckks_clear_sample(x.requires_grad_(), u), ValueError)):
        with pytest.raises(error):
            call()
    assert K.ckks_clear_sample(torch.zeros(0, 50, device="cuda"), u[:0]).shape == (0,)
