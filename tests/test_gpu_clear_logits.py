"""Rules on logits against 64 bits, entry by entry."""
import math

import numpy as np
import pytest
import torch

from tests.clear_util import TINY, TYPES, U, close, gen, randn

pytestmark = pytest.mark.gpu


def make(rows, vocab, dtype, seed, hist=20, biases=5, mask=True, lo=0, hi=None):
    g, host = gen(seed), np.random.default_rng(seed)
    s = {"logits": 3 * randn(g, rows, vocab)}
    s["logits"] = s["logits"].to(dtype)
    if hist:
        n = host.integers(0, hist + 1, rows)
        n[0] = hist
        s["tokens"] = torch.from_numpy(host.integers(lo, vocab if hi is None else hi, n.sum()).astype(np.int32)).cuda()
        s["token_start"] = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda()
        s["n_prompt"] = torch.from_numpy((n // 2).astype(np.int32)).cuda()
        s["repetition"], s["frequency"], s["presence"] = (
            a + b * torch.rand(rows, generator=g, device="cuda") for a, b in ((0.8, 0.9), (-0.3, 1), (-0.3, 1)))
    if biases:
        n = host.integers(0, biases + 1, rows)
        s["bias_ids"] = torch.from_numpy(host.integers(lo, vocab if hi is None else hi, n.sum()).astype(np.int32)).cuda()
        s["bias"] = 5 * randn(g, int(n.sum()))
        s["bias_start"] = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda()
    if mask:
        s["mask"] = torch.from_numpy(host.integers(-2**31, 2**31, (rows, (vocab + 31) // 32)).astype(np.int32)).cuda()
    return s


def reference(s):
    """(result, bound) in 64 bits: up to six roundings of 32 bits on terms of the sizes summed in the bound."""
    l = s["logits"].double().cpu().numpy().copy()
    size = np.abs(l)
    rows, vocab = l.shape
    cpu = {k: v.cpu().numpy() for k, v in s.items() if k != "logits"}
    for r in range(rows):
        if "token_start" in cpu:
            a, b = cpu["token_start"][r], cpu["token_start"][r + 1]
            words = cpu["tokens"][a:b]
            made = words[cpu["n_prompt"][r] if "n_prompt" in cpu else 0:]
            rep, freq, pres = (float(cpu[k][r]) if k in cpu else d for k, d in (("repetition", 1.0), ("frequency", 0.0), ("presence", 0.0)))
            for v in set(int(w) for w in words if 0 <= w < vocab):
                count = int((made == v).sum())
                l[r, v] = l[r, v] / rep if l[r, v] > 0 else l[r, v] * rep
                size[r, v] = abs(l[r, v]) + abs(freq) * count + abs(pres)
                l[r, v] -= freq * count + (pres if count else 0.0)
        if "bias_start" in cpu:
            last = {}
            for i in range(cpu["bias_start"][r], cpu["bias_start"][r + 1]):
                last[int(cpu["bias_ids"][i])] = float(cpu["bias"][i])
            for v, x in last.items():
                if 0 <= v < vocab:
                    l[r, v] += x
                    size[r, v] += abs(x)
    if "mask" in cpu:
        v = np.arange(vocab)
        l[(cpu["mask"][:, v >> 5] >> (v & 31)) & 1 == 0] = -math.inf
    return torch.from_numpy(l).cuda(), torch.from_numpy(size).cuda()


def check(s, out=None):
    from paper_2604_09975_amd import clear as K
    want, size = reference(s)
    kept = {k: v.clone() for k, v in s.items()}
    got = K.ckks_clear_logits(**s, out=out)
    # what the type cannot hold is infinite in it
    want = torch.where(torch.isfinite(want) & (want.abs() > torch.finfo(got.dtype).max), torch.sign(want) * math.inf, want)
    u = U[got.dtype]
    fine = torch.where(torch.isfinite(want), want.abs(), 0.0)
    close(got, want, u * fine + 2.0**-21 * torch.nan_to_num(size, posinf=0.0) + TINY[got.dtype])
    if out is not s["logits"]:
        assert all(torch.equal(s[k].nan_to_num(), kept[k].nan_to_num()) for k in s)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 5, 32, 33, 2047, 2049, 8192, 8193, 50257])
def test_against_64_bits(vocab, dtype):
    for rows in (1, 3):
        check(make(rows, vocab, TYPES[dtype], vocab + rows, hist=200, biases=30))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows(dtype):
    check(make(130, 17001, TYPES[dtype], 9, hist=300, biases=20))


@pytest.mark.parametrize("parts", [(0, 0, False), (9, 0, False), (0, 9, False), (9, 9, False), (0, 0, True), (9, 0, True), (0, 9, True)])
def test_each_rule_alone(parts):
    for rows, vocab in ((2, 3000), (300, 9000)):
        check(make(rows, vocab, torch.float16, 4, *parts))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,biases", [(3, 2100, 4000), (2, 9000, 12000), (1, 40, 600), (257, 1500, 1400), (257, 300, 520)])
def test_more_biases_than_a_table_holds(rows, vocab, biases, dtype):
    """A bias for most tokens, several for some; rows with few beside rows with many."""
    check(make(rows, vocab, TYPES[dtype], rows + vocab, hist=60, biases=biases))


def test_one_token_many_times_and_the_last_bias_counts():
    s = make(4, 700, torch.float32, 5, hist=5000, biases=400, lo=3, hi=9)
    check(s)
    for k in ("repetition", "frequency", "presence", "n_prompt"):
        t = dict(s)
        del t[k]
        check(t)


def test_ids_outside_the_vocabulary():
    s = make(3, 900, torch.bfloat16, 6, hist=100, biases=50, lo=-200, hi=1100)
    check(s)


def test_rows_that_the_mask_leaves_empty_infinities_and_nan():
    s = make(5, 1000, torch.float32, 7, hist=50, biases=10)
    s["mask"][1] = 0
    s["mask"][2] = -1
    s["logits"][2, 10], s["logits"][2, 11], s["logits"][2, 12] = math.inf, -math.inf, math.nan
    s["logits"][1, 3] = math.nan                       # masked: gone
    s["logits"][3] = torch.finfo(torch.float32).min    # the type's lowest value is no mask
    s["mask"][3] = -1
    want_finite = {k: v.clone() for k, v in s.items()}
    got = check(want_finite)
    assert (got[1] == -math.inf).all() and torch.isnan(got[2, 12])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_wider_output_places_and_strides(dtype):
    from paper_2604_09975_amd import clear as K
    s = make(6, 5001, TYPES[dtype], 8)
    plain = check(s)
    wide = torch.empty(6, 5001, device="cuda")
    assert check(s, out=wide) is wide
    assert torch.equal(wide.to(plain.dtype), plain)
    t = dict(s, logits=s["logits"].clone())
    assert check(t, out=t["logits"]) is t["logits"] and torch.equal(t["logits"], plain)
    # rows of a wider array at an odd place; the mask's rows padded
    room = torch.zeros(6, 6001, dtype=TYPES[dtype], device="cuda")
    room[:, 3:5004] = s["logits"]
    out = torch.zeros(6, 7001, dtype=TYPES[dtype], device="cuda")
    pad = torch.zeros(6, 200, dtype=torch.int32, device="cuda")
    pad[:, :157] = s["mask"]
    K.ckks_clear_logits(**dict(s, logits=room[:, 3:5004], mask=pad), out=out[:, 1:5002])
    assert torch.equal(out[:, 1:5002], plain) and not out[:, 0].any() and not out[:, 5002:].any()
    one = {k: s[k] for k in ("logits",)}
    assert torch.equal(K.ckks_clear_logits(one["logits"][0]), one["logits"][0])


def test_no_rows_and_empty_lists():
    from paper_2604_09975_amd import clear as K
    assert K.ckks_clear_logits(torch.empty(0, 50, device="cuda")).shape == (0, 50)
    x = randn(gen(1), 2, 50)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    start = torch.zeros(3, dtype=torch.int32, device="cuda")
    y = K.ckks_clear_logits(x, tokens=none, token_start=start, presence=torch.ones(2, device="cuda"),
                            bias_ids=none, bias=none.float(), bias_start=start)
    assert torch.equal(x, y)


def test_refusals():
    from paper_2604_09975_amd import binding as B
    from paper_2604_09975_amd import clear as K
    s = make(3, 500, torch.float16, 2)
    with pytest.raises(B.CkksError):
        K.ckks_clear_logits(s["logits"], presence=s["presence"])
    with pytest.raises(B.CkksError):
        K.ckks_clear_logits(s["logits"], bias=s["bias"], bias_ids=s["bias_ids"])
    with pytest.raises(ValueError):
        K.ckks_clear_logits(s["logits"], mask=s["mask"][:, :15])
    with pytest.raises(ValueError):
        K.ckks_clear_logits(**dict(s, token_start=s["token_start"][:3]))
    with pytest.raises(ValueError):
        K.ckks_clear_logits(**dict(s, bias=s["bias"][:-1]))
    with pytest.raises(TypeError):
        K.ckks_clear_logits(**dict(s, tokens=s["tokens"].long()))
    with pytest.raises(B.CkksError):
        K.ckks_clear_logits(s["logits"], out=torch.empty(3, 500, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(B.CkksError):
        room = torch.empty(4, 500, dtype=torch.float16, device="cuda")
        K.ckks_clear_logits(room[:3], out=room[1:])
