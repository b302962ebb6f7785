"""The steps in the clear on other streams than the default, and captured into a graph whose lengths and values change between
the replays."""
import pytest
import torch

from tests.clear_util import Cache, gen, randn

pytestmark = pytest.mark.gpu


def step(K, s):
    """A token's way: norm, append with rotation, attention split over blocks, norm's gradient, rules."""
    c = s["cache"]
    y, mean, rstd = K.ckks_clear_layer_norm(s["x"], s["w"], s["b"])
    q = K.ckks_clear_cache_append(s["k"], s["v"], *c.args(), cos=s["cos"], sin=s["sin"], q=s["q"])
    a = K.ckks_clear_attend(q, *c.args())
    grads = K.ckks_clear_layer_norm_grad(s["dy"], s["x"], mean, rstd, s["w"])
    l = K.ckks_clear_logits(s["logits"], tokens=s["tokens"], token_start=s["start"], frequency=s["freq"], mask=s["mask"])
    return (y, q, a, l, c.k.clone(), c.v.clone()) + tuple(grads)


def make(seed):
    g = gen(seed)
    c = Cache([(1, 2500), (3, 900), (1, 1)], 8, 2, 64, 16, torch.bfloat16, seed, width=160)
    used = torch.randperm(c.k.shape[0], generator=torch.Generator().manual_seed(seed))
    c.table[:, :] = used[torch.arange(3 * 160) % c.k.shape[0]].view(3, 160).to(torch.int32)
    c.page_table.copy_(c.table)
    angle = torch.rand(160 * 16, 32, generator=g, device="cuda")
    return {"cache": c, "x": randn(g, 40, 600, dtype=torch.bfloat16), "dy": randn(g, 40, 600, dtype=torch.bfloat16),
            "w": randn(g, 600), "b": randn(g, 600), "q": randn(g, 5, 8, 64, dtype=torch.bfloat16), "k": randn(g, 5, 2, 64, dtype=torch.bfloat16),
            "v": randn(g, 5, 2, 64, dtype=torch.bfloat16), "cos": angle.cos(), "sin": angle.sin(),
            "logits": randn(g, 3, 5000), "tokens": torch.randint(0, 5000, (90,), generator=g, device="cuda", dtype=torch.int32),
            "start": torch.tensor([0, 30, 30, 90], dtype=torch.int32, device="cuda"), "freq": torch.rand(3, generator=g, device="cuda"),
            "mask": torch.randint(-2**31, 2**31 - 1, (3, 157), generator=g, device="cuda", dtype=torch.int32)}


def refill(s, t):
    """The values and lengths of t in the tensors of s."""
    for k, v in t.items():
        if k != "cache":
            s[k].copy_(v)
    for k in ("k", "v", "page_table", "kv_len"):
        getattr(s["cache"], k).copy_(getattr(t["cache"], k))


def test_on_another_stream():
    from paper_2604_09975_amd import clear as K
    want = step(K, make(1))
    s = make(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)          # what the calls read is written late on their own stream
        s["x"].mul_(1)
        got = step(K, s)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_captured_and_replayed():
    from paper_2604_09975_amd import clear as K
    s = make(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(K, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    refill(s, make(2))
    with torch.cuda.graph(graph, stream=side):
        got = step(K, s)
    lengths = ([2500, 900, 1], [2, 2500, 77], [512, 3, 2000], [1, 3, 1])
    for seed, lens in zip((2, 3, 4, 5), lengths):
        t, u = make(seed), make(seed)
        for x in (t, u):
            x["cache"].kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        refill(s, t)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = step(K, u)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), seed
