"""A key holder's cache in 8 bits and the choice of the next token: what they compute and how long they take.

Between two encrypted projections the key holder keeps keys and values of a conversation in pages, attends over them and, at the
end of a step, draws a token from the logits.  Here the pages hold one byte for each entry and a power of two for each 32
of a head's entries.  Four operators: new tokens into such pages, their queries and keys normed and rotated on the way
("store", which also reads the new rows back: what the cache holds of them); attention over the pages ("attend"); a conversation's
rows out of them ("read"); and the draw ("sample").  `own` false: written out in elementary torch operations; `own` true: the
framework's calls.

Rounding to 8 bits and the order of sums next to the border of two tokens decide about whole steps of a result: what leads there
is computed in 64 bits.  Lengths of a ragged batch follow from the case alone (`lengths`), the values from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
LARGEST = {"e4m3": 448.0, "i8": 127.0}
BLOCK = 32       # entries of a head that share a power of two
LEAST = -100     # the smallest power of two of a block


def listed():
    return [
        # one new token of each of 32 conversations with learned positions: no rotation, latency only
        {"name": "store_token", "kind": "store", "seqs": 32, "new": 1, "old": 700, "heads": 12, "kv_heads": 12, "dim": 64,
         "page": 16, "rot": 0, "interleaved": False, "norm": False, "format": "i8", "dtype": "f16", "spread": 1},
        # prompts of eight conversations, queries and keys normed for each head and rotated, heads shared four to one
        {"name": "store_prompt", "kind": "store", "seqs": 8, "new": 4096, "old": 1000, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "rot": 128, "interleaved": False, "norm": True, "format": "e4m3", "dtype": "bf16", "spread": 2},
        # decoded values in 32 bits, heads of an odd width, half of each rotated in pairs side by side
        {"name": "store_ragged", "kind": "store", "seqs": 5, "new": 777, "old": 1303, "heads": 8, "kv_heads": 4, "dim": 80,
         "page": 32, "rot": 40, "interleaved": True, "norm": True, "format": "i8", "dtype": "f32", "spread": 3},
        # one token of one conversation after a segment: the smallest call of a decoding loop
        {"name": "attend_token", "kind": "attend", "seqs": 1, "new": 1, "old": 127, "heads": 12, "kv_heads": 12, "dim": 64,
         "page": 16, "causal": True, "window": 0, "format": "i8", "dtype": "bf16", "spread": 0},
        # a decoding step of 64 conversations of very different lengths
        {"name": "attend_batch", "kind": "attend", "seqs": 64, "new": 1, "old": 8191, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "causal": True, "window": 0, "format": "e4m3", "dtype": "bf16", "spread": 3},
        # a decoding step over one long document, as decryption yields it: few rows, a long axis
        {"name": "attend_long", "kind": "attend", "seqs": 1, "new": 1, "old": 131001, "heads": 16, "kv_heads": 2, "dim": 128,
         "page": 256, "causal": True, "window": 0, "format": "i8", "dtype": "f32", "spread": 0},
        # two prompts taken in by chunks, the chunk's tokens over all that came before: the largest products
        {"name": "attend_prompt", "kind": "attend", "seqs": 2, "new": 4096, "old": 12301, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "causal": True, "window": 0, "format": "e4m3", "dtype": "bf16", "spread": 4},
        # one conversation's rows out of the cache, to be encrypted or kept elsewhere
        {"name": "read_segment", "kind": "read", "seqs": 1, "new": 128, "old": 0, "kv_heads": 12, "dim": 64, "page": 16,
         "format": "i8", "dtype": "f32", "spread": 0},
        # sixteen conversations move out
        {"name": "read_batch", "kind": "read", "seqs": 16, "new": 8001, "old": 100, "kv_heads": 8, "dim": 128, "page": 64,
         "format": "e4m3", "dtype": "bf16", "spread": 5},
        # the next token of one conversation, odd vocabulary
        {"name": "sample_token", "kind": "sample", "rows": 1, "vocab": 50257, "top_k": 50, "top_p": 0.95, "min_p": 0.0,
         "dtype": "f32", "spread": 0},
        # a step of 256 conversations with a large vocabulary, each with settings of its own
        {"name": "sample_batch", "kind": "sample", "rows": 256, "vocab": 131072, "top_k": 0, "top_p": 0.9, "min_p": 0.02,
         "dtype": "bf16", "spread": 6},
        # as many without any limit: every token counts
        {"name": "sample_all", "kind": "sample", "rows": 64, "vocab": 120001, "top_k": 0, "top_p": 1.0, "min_p": 0.0,
         "dtype": "f32", "spread": 7},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(("store", "store", "attend", "attend", "attend", "read", "sample", "sample"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    case = {"kind": kind, "dtype": dtype, "spread": rng.randrange(1, 1 << 30)}
    if kind == "sample":
        vocab = _spread(rng, 1000, 131072)
        rows = _spread(rng, 1, min(512, 256 * 131072 // (2 if dtype == "f32" else 1) // vocab))
        return {**case, "rows": rows, "vocab": vocab, "top_k": rng.choice((0, _spread(rng, 1, 1000))),
                "top_p": rng.choice((1.0, rng.uniform(0.3, 0.99))), "min_p": rng.choice((0.0, rng.uniform(0.01, 0.3)))}
    dim = rng.choice((64, 64, 80, 96, 128, 128))
    kv_heads = rng.choice((1, 2, 4, 8, 12))
    heads = kv_heads * rng.choice((1, 1, 2, 4, 8) if kv_heads < 8 else (1, 2, 4) if kv_heads == 8 else (1,))
    case.update(kv_heads=kv_heads, dim=dim, page=rng.choice((16, 32, 64, 128, 256)), format=rng.choice(("e4m3", "i8")))
    if kind == "read":
        seqs = _spread(rng, 1, 32)
        return {**case, "seqs": seqs, "new": _spread(rng, 1, min(8192, 65536 // seqs)), "old": rng.choice((0, _spread(rng, 1, 500)))}
    case["heads"] = heads
    if kind == "store":
        seqs = _spread(rng, 1, 64)
        new = rng.choice((1, _spread(rng, 1, min(4096, 16384 // seqs))))
        return {**case, "seqs": seqs, "new": new, "old": _spread(rng, 1, 2000), "rot": rng.choice((0, dim // 2, dim, dim)),
                "interleaved": rng.random() < 0.3, "norm": rng.random() < 0.6}
    case.update(causal=rng.random() < 0.85, window=0)
    if rng.random() < 0.6:  # decoding: a token or a few for each sequence
        seqs = _spread(rng, 1, 64)
        new = rng.choice((1, 1, rng.randrange(2, 9)))
        old = _spread(rng, 1, min(131001, 64 * 8191 // seqs // (2 if dtype == "f32" else 1)))
    else:  # a chunk of a prompt
        new = _spread(rng, 9, 2048)
        seqs = _spread(rng, 1, max(1, min(16, 4096 // new)))
        old = rng.choice((0, _spread(rng, 1, 8192)))
        if dtype == "f32":
            new, old = max(1, new // 2), old // 4
    if case["causal"] and rng.random() < 0.25:
        case["window"] = _spread(rng, 16, 4096)
    return {**case, "seqs": seqs, "new": new, "old": old}


def lengths(case):
    """(new tokens, tokens in the cache with them) of each sequence: `new` and `old` are the most; `spread` 0: all have that."""
    rng = random.Random(case["spread"])
    got = []
    for b in range(case["seqs"]):
        n, old = case["new"], case["old"]
        if case["spread"] and b:
            n, old = rng.randint(max(1, n // 2), n), rng.randint(old // 16, old)
        got.append((n, n + old))
    return got


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, to=None):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(to or dtype)

    s = {"kind": case["kind"], "case": case}
    if case["kind"] == "sample":
        rows, rng = case["rows"], random.Random(case["spread"])
        s["logits"] = (normal(rows, case["vocab"], to=torch.float32) * 2.5).to(dtype)
        s["u"] = torch.rand(rows, generator=g, device="cuda")
        one = not case["spread"]

        def settings(at):  # each conversation's own, around the case's
            return torch.tensor([at(1.0 if one else rng.uniform(0.6, 1.4)) for _ in range(rows)], device="cuda")
        s["temperature"] = settings(lambda f: 0.8 * f)
        if case["top_k"]:
            s["top_k"] = settings(lambda f: max(1, int(case["top_k"] * f))).to(torch.int32)
        if case["top_p"] < 1:
            s["top_p"] = settings(lambda f: 1 - (1 - case["top_p"]) * f)
        if case["min_p"]:
            s["min_p"] = settings(lambda f: case["min_p"] * f)
        return s
    lens = lengths(case)
    kv_heads, dim, page = case["kv_heads"], case["dim"], case["page"]
    total = sum(n for n, _ in lens)
    need = [-(-kv // page) for _, kv in lens]
    n_pages = sum(need) + 3
    order = np.random.default_rng(seed).permutation(n_pages)[:sum(need)]
    table = np.full((len(lens), max(need)), -1, np.int32)  # places that no sequence reaches hold no page
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    s["page_table"] = torch.from_numpy(table).cuda()
    s["q_start"] = torch.tensor(np.concatenate([[0], np.cumsum([n for n, _ in lens])]), dtype=torch.int32, device="cuda")
    s["kv_len"] = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device="cuda")
    s["total"] = total
    shape, blocks = (n_pages, kv_heads, page, dim), -(-dim // BLOCK)
    for x in "kv":
        # codes of values of about the size 1: a block's largest fills its range, the power of two differs by one or so
        top = LARGEST[case["format"]] / 2.5
        code = (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * (top / 2)).clamp_(-2 * top, 2 * top)
        s[x + "_pages"] = (code.round_() if case["format"] == "i8" else code).to(CODES[case["format"]])
        e = torch.randint(-1, 2, (n_pages, kv_heads, page, blocks), generator=g, device="cuda")
        s[x + "_scale"] = (e + 127 - int(math.log2(top / 2))).to(torch.uint8)
    if case["kind"] == "read":
        return s
    heads = case["heads"]
    if case["kind"] == "attend":
        s["q"] = normal(total, heads, dim) * (1.0 if case["spread"] % 2 else 1.5)
        return s
    # queries, keys and values as the columns of one decrypted projection
    qkv = normal(total, (heads + 2 * kv_heads) * dim)
    s["q"] = qkv[:, :heads * dim].view(total, heads, dim)
    s["k"] = qkv[:, heads * dim:(heads + kv_heads) * dim].view(total, kv_heads, dim)
    s["v"] = qkv[:, (heads + kv_heads) * dim:].view(total, kv_heads, dim)
    if case["norm"]:
        s["q_norm"], s["k_norm"] = 1 + 0.1 * normal(dim, to=torch.float32), 1 + 0.1 * normal(dim, to=torch.float32)
    if case["rot"]:
        # the program's table of angles, one row for every position that the cache can hold
        angle = torch.arange(max(need) * page, device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2604_09975_amd import clear as K
    if s["kind"] == "sample":
        prob = torch.empty_like(s["u"])
        token = K.ckks_clear_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s.get("top_k"), top_p=s.get("top_p"),
                                    min_p=s.get("min_p"), prob=prob)
        return token, prob
    cache = (s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["page_table"], s["q_start"], s["kv_len"])
    case = s["case"]
    if s["kind"] == "attend":
        return K.ckks_clear_packed_attend(s["q"], *cache, causal=case["causal"], window=case["window"])
    if s["kind"] == "read":
        return K.ckks_clear_packed_read(*cache, s["total"], DTYPES[case["dtype"]])
    q = K.ckks_clear_packed_append(s["k"], s["v"], *cache, cos=s.get("cos"), sin=s.get("sin"), interleaved=case["interleaved"], q=s["q"],
                                   k_norm=s.get("k_norm"), q_norm=s.get("q_norm"), eps=1e-6)
    return (q,) + tuple(K.ckks_clear_packed_read(*cache, s["total"], s["k"].dtype))


def _run_plain(s):
    return {"store": _plain_store, "attend": _plain_attend, "read": _plain_read, "sample": _plain_sample}[s["kind"]](s)


def _plain_sample(s):
    l = s["logits"].double()
    rows, vocab = l.shape
    # largest first, of equal ones the lowest index; weights against the largest, which is 1
    l, ids = torch.sort(l, dim=1, descending=True, stable=True)
    w = torch.exp((l - l[:, :1]) / s["temperature"].double()[:, None])
    rank = torch.arange(vocab, device=l.device)
    if "top_k" in s:
        w = torch.where(rank < s["top_k"][:, None], w, 0.0)
    keep = w > 0
    if "top_p" in s:
        before = w.cumsum(1) - w
        keep = keep & ((before < s["top_p"].double()[:, None] * w.sum(1, keepdim=True)) | (rank == 0))
    if "min_p" in s:
        keep = keep & (w >= s["min_p"].double()[:, None])
    w = torch.zeros_like(w).scatter_(1, ids, torch.where(keep, w, 0.0))
    upto = w.cumsum(1)
    total = upto[:, -1:]
    token = (upto <= s["u"].double()[:, None] * total).sum(1, keepdim=True).clamp_(max=vocab - 1)
    return token[:, 0].int(), (w.gather(1, token) / total)[:, 0].float()


def _token_places(s):
    """Sequence and cache position of each new token."""
    start = s["q_start"].long()
    at = torch.arange(s["total"], device=start.device)
    seq = torch.searchsorted(start, at, right=True) - 1
    return seq, s["kv_len"].long()[seq] - (start[seq + 1] - at)


def _power(e):
    """2^e of whole numbers, to the last bit."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _values(codes, scale):
    """What codes [..., dim] with powers of two [..., blocks] stand for, in 32 bits."""
    power = _power(scale.int() - 127).float().repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]
    return codes.float() * power


def _plain_rotate(x, cos, sin, interleaved):
    h = cos.shape[-1]
    c, n = cos.double()[:, None], sin.double()[:, None]
    if interleaved:
        a, b = x[..., 0:2 * h:2], x[..., 1:2 * h:2]
        r = torch.stack((a * c - b * n, b * c + a * n), -1).flatten(-2)
    else:
        a, b = x[..., :h], x[..., h:2 * h]
        r = torch.cat((a * c - b * n, b * c + a * n), -1)
    return torch.cat((r, x[..., 2 * h:]), -1)


def _plain_pack(x, form):
    """Codes and powers of two of 64-bit values [..., dim]."""
    dim = x.shape[-1]
    blocks = -(-dim // BLOCK)
    x = torch.nn.functional.pad(x, (0, blocks * BLOCK - dim)).unflatten(-1, (blocks, BLOCK))
    # the smallest power with largest <= LARGEST * 2^e
    m, e = torch.frexp(x.abs().amax(-1) / LARGEST[form])
    e = torch.where(m == 0.5, e - 1, e)
    e = torch.where(m == 0, LEAST, e).clamp_(min=LEAST)
    x = x * _power(-e[..., None])
    if form == "e4m3":  # four significant bits, down to steps of 2^-9
        step = _power((torch.frexp(x)[1] - 4).clamp_(min=-9))
        x = torch.round(x / step) * step
    else:
        x = torch.round(x)
    return x.flatten(-2)[..., :dim].float().to(CODES[form]), (e + 127).to(torch.uint8)


def _plain_store(s):
    seq, pos = _token_places(s)
    page, case = s["k_pages"].shape[2], s["case"]
    where, row = s["page_table"][seq, pos // page].long(), pos % page
    q, k = s["q"].double(), s["k"].double()
    if "q_norm" in s:
        q, k = (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.double() for x, w in ((q, s["q_norm"]), (k, s["k_norm"])))
    if "cos" in s:
        q, k = (_plain_rotate(x, s["cos"][pos], s["sin"][pos], case["interleaved"]) for x in (q, k))
    got = []
    for name, x in (("k", k), ("v", s["v"].double())):
        codes, scale = _plain_pack(x, case["format"])
        s[name + "_pages"].view(torch.uint8)[where, :, row] = codes.view(torch.uint8)
        s[name + "_scale"][where, :, row] = scale
        got.append(_values(s[name + "_pages"].view(torch.uint8)[where, :, row].view(codes.dtype), s[name + "_scale"][where, :, row]).to(s["k"].dtype))
    return q.to(s["q"].dtype), got[0], got[1]


def _plain_read(s):
    seq, pos = _token_places(s)
    page, to = s["k_pages"].shape[2], DTYPES[s["case"]["dtype"]]
    where, row = s["page_table"][seq, pos // page].long(), pos % page
    k, v = (_values(s[x + "_pages"].view(torch.uint8)[where, :, row].view(s[x + "_pages"].dtype), s[x + "_scale"][where, :, row]).to(to) for x in "kv")
    return k, v


def _plain_attend(s):
    case = s["case"]
    q, table = s["q"], s["page_table"].clamp(min=0).long()
    seqs, heads, dim = case["seqs"], case["heads"], case["dim"]
    kv_heads, page = s["k_pages"].shape[1], case["page"]
    group, span = heads // kv_heads, table.shape[1] * page
    seq, pos = _token_places(s)
    slot = torch.arange(q.shape[0], device=q.device) - s["q_start"].long()[seq]
    most = case["new"]
    # padded to the longest: queries [seq, kv head, token * group, dim], keys [seq, kv head, dim, position]
    qp = torch.zeros(seqs, most, heads, dim, device=q.device)
    qp[seq, slot] = q.float()
    qp = qp.view(seqs, most, kv_heads, group, dim).transpose(1, 2).reshape(seqs, kv_heads, most * group, dim)
    k = _values(s["k_pages"], s["k_scale"])[table].permute(0, 2, 4, 1, 3).reshape(seqs, kv_heads, dim, span)
    v = _values(s["v_pages"], s["v_scale"])[table].permute(0, 2, 1, 3, 4).reshape(seqs, kv_heads, span, dim)
    score = torch.matmul(qp, k).mul_(dim ** -0.5).view(seqs, kv_heads, most, group, span)
    t = torch.zeros(seqs, most, dtype=torch.long, device=q.device)
    t[seq, slot] = pos
    j = torch.arange(span, device=q.device)
    seen = (j < s["kv_len"].long()[:, None, None]).expand(seqs, most, span)
    if case["causal"]:
        seen = seen & (j <= t[..., None])
        if case["window"]:
            seen = seen & (j > t[..., None] - case["window"])
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    score.sub_(score.amax(-1, keepdim=True).clamp_(min=-3e38)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(seqs, kv_heads, most * group, span), v).view(seqs, kv_heads, most, group, dim)
    out = torch.where(total > 0, out / total, 0.0).transpose(1, 2).reshape(seqs, most, heads, dim)
    return out[seq, slot].to(q.dtype)


def _pairs(case):
    """Pairs of a query token and a key that it sees."""
    n = 0
    for new, kv in lengths(case):
        if not case["causal"]:
            n += new * kv
            continue
        first, w = kv - new, case["window"]
        if not w:
            n += new * (first + 1) + new * (new - 1) // 2
        else:
            n += sum(min(w, t + 1) for t in range(first, kv))
    return n


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "sample":
        cells = case["rows"] * case["vocab"]
        return {"bytes": cells * e + 28 * case["rows"], "flops": 6 * cells}
    total = sum(n for n, _ in lengths(case))
    dim, kv_heads = case["dim"], case["kv_heads"]
    packed = dim + -(-dim // BLOCK)  # bytes of a row of the cache
    if case["kind"] == "read":
        return {"bytes": 2 * total * kv_heads * (packed + dim * e), "flops": 2 * total * kv_heads * dim}
    heads = case["heads"]
    if case["kind"] == "store":
        # the new rows in, queries out, codes and powers out, and what the cache holds of them out
        moved = total * (heads + 2 * kv_heads) * dim * e + total * heads * dim * e + 2 * total * kv_heads * (packed + dim * e)
        places = set().union(*(range(kv - n, kv) for n, kv in lengths(case))) if case["rot"] else ()
        return {"bytes": moved + 4 * case["rot"] * len(places), "flops": total * ((heads + kv_heads) * (3 * case["rot"] + (4 * dim if case["norm"] else 0)) + 8 * kv_heads * dim)}
    w = case["window"]
    kept = sum(min(kv, new + w - 1) if w else kv for new, kv in lengths(case))
    return {"bytes": 2 * total * heads * dim * e + 2 * kept * kv_heads * packed, "flops": 4 * dim * heads * _pairs(case)}


def _exact_powers():
    """2^-160 .. 2^160."""
    return torch.tensor([2.0 ** k for k in range(-160, 161)], dtype=torch.float64, device="cuda")


def _exact_code_values(form):
    """The values of 8 bits without a sign, rising; their place is even where the last bit of the code is 0."""
    if form == "i8":
        return torch.arange(128, dtype=torch.float64, device="cuda")
    n = torch.arange(127, device="cuda")  # the last pattern is no number
    e, m = n // 8, (n % 8).double()
    return torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * _exact_powers()[e - 7 + 160])


def _exact_pack(x, form):
    """64-bit values [rows][dim] as the cache holds them: the nearest of the values that 8 bits have, block by block."""
    grid, powers = _exact_code_values(form), _exact_powers()
    middle = (grid[1:] + grid[:-1]) / 2
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], BLOCK):
        y = x[:, c:c + BLOCK]
        top = y.abs().max(1, keepdim=True).values
        power = powers[160 + LEAST + (top > grid[-1] * powers[160 + LEAST:]).sum(1, keepdim=True)]
        size = y.abs() / power
        at = torch.searchsorted(middle, size.contiguous())
        tie = (at < len(middle)) & (middle[at.clamp(max=len(middle) - 1)] == size) & (at % 2 == 1)
        out[:, c:c + BLOCK] = torch.copysign(grid[at + tie.long()] * power, y)
    return out


def _exact_rows(case, s, which, b, h, kv):
    """The first kv keys or values of one sequence and head, in 64 bits."""
    page = case["page"]
    pages = s["page_table"][b, :-(-kv // page)].long()
    codes = s[which + "_pages"].view(torch.uint8)[pages, h].view(s[which + "_pages"].dtype).reshape(-1, case["dim"])[:kv].to(torch.float32).double()
    power = _exact_powers()[s[which + "_scale"][pages, h].reshape(codes.shape[0] + (-kv) % page, -1)[:kv].long() + 160 - 127]
    for c in range(power.shape[1]):
        codes[:, c * BLOCK:(c + 1) * BLOCK] *= power[:, c:c + 1]
    return codes


def exact(case, seed):
    """The operator's definition in 64 bits, one sequence and one head (one row) after the other."""
    s = prepare(case, seed)
    wide = torch.float64
    if case["kind"] == "sample":
        token, prob = [], []
        for r in range(case["rows"]):
            l = s["logits"][r].to(wide)
            p = torch.softmax(l / s["temperature"][r].to(wide), 0)
            order = torch.argsort(l, descending=True, stable=True)
            if "top_k" in s:
                order = order[:int(s["top_k"][r])]
            have = p[order] / p[order].sum()
            if "top_p" in s:
                sums = have.cumsum(0)
                have = have[:1 + int((sums[:-1] < s["top_p"][r].to(wide)).sum())]
            if "min_p" in s:
                have = have[have >= s["min_p"][r].to(wide) * have[0]]
            kept = torch.sort(order[:len(have)]).values
            share = p[kept] / p[kept].sum()
            at = min(int((share.cumsum(0) <= s["u"][r].to(wide)).sum()), len(kept) - 1)
            token.append(int(kept[at]))
            prob.append(float(share[at]))
        return torch.tensor(token, dtype=torch.int32), torch.tensor(prob, dtype=wide)
    lens = lengths(case)
    kv_heads, dim = case["kv_heads"], case["dim"]
    if case["kind"] == "read":
        out = torch.empty(2, s["total"], kv_heads, dim, dtype=wide, device="cuda")
        at = 0
        for b, (n, kv) in enumerate(lens):
            for h in range(kv_heads):
                for i, which in enumerate("kv"):
                    out[i, at:at + n, h] = _exact_rows(case, s, which, b, h, kv)[kv - n:]
            at += n
        return out[0], out[1]
    if case["kind"] == "store":
        new, half, at = {x: s[x].to(wide) for x in "qkv"}, case["rot"] // 2, 0
        if case["norm"]:
            for x in "qk":
                length = torch.linalg.vector_norm(new[x], dim=-1, keepdim=True)
                new[x] = new[x] / torch.sqrt(length ** 2 / dim + 1e-6) * s[x + "_norm"].to(wide)
        for n, kv in lens:
            if half:
                angle = torch.complex(s["cos"][kv - n:kv].to(wide), s["sin"][kv - n:kv].to(wide))[:, None]
                one = slice(0, 2 * half, 2) if case["interleaved"] else slice(0, half)
                two = slice(1, 2 * half, 2) if case["interleaved"] else slice(half, 2 * half)
                for x in "qk":
                    y = new[x][at:at + n]
                    z = torch.complex(y[..., one].clone(), y[..., two].clone()) * angle
                    y[..., one], y[..., two] = z.real, z.imag
            at += n
        return (new["q"],) + tuple(_exact_pack(new[x].reshape(-1, dim), case["format"]).view(-1, kv_heads, dim) for x in "kv")
    out = torch.zeros(s["q"].shape, dtype=wide, device="cuda")
    at, group = 0, case["heads"] // kv_heads
    for b, (n, kv) in enumerate(lens):
        t = torch.arange(kv - n, kv, device="cuda")[:, None]
        j = torch.arange(kv, device="cuda")[None]
        hidden = torch.zeros(n, kv, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden = j > t
            if case["window"]:
                hidden = hidden | (j + case["window"] <= t)
        for g in range(kv_heads):
            k, v = (_exact_rows(case, s, which, b, g, kv) for which in "kv")
            for h in range(g * group, (g + 1) * group):
                p = torch.mm(s["q"][at:at + n, h].to(wide), k.t().contiguous()) / math.sqrt(dim)
                p = torch.softmax(p.masked_fill(hidden, -math.inf), dim=1)
                out[at:at + n, h] = torch.mm(p, v)
        at += n
    return out
