"""The steps in the clear beside torch's autograd: no gradient is lost without a word, and what is written in place is noticed."""
import pytest
import torch

from tests.clear_util import Cache, gen, randn

pytestmark = pytest.mark.gpu


def calls(K):
    """(name, call of named tensors, the tensors, those of them that may require a gradient, those that are written)."""
    g = gen(1)
    c = Cache([(4, 20)], 4, 2, 64, 16, torch.float16, 1)
    x, w, b, dy = randn(g, 6, 64), randn(g, 64), randn(g, 64), randn(g, 6, 64)
    _, mean, rstd = K.ckks_clear_layer_norm(x, w, b)
    page = dict(k_pages=c.k, v_pages=c.v, page_table=c.page_table, q_start=c.q_start, kv_len=c.kv_len)
    new = dict(k=randn(g, 4, 2, 64, dtype=torch.float16), v=randn(g, 4, 2, 64, dtype=torch.float16))
    words = dict(tokens=torch.zeros(3, dtype=torch.int32, device="cuda"), token_start=torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda"),
                 bias_ids=torch.zeros(1, dtype=torch.int32, device="cuda"), bias_start=torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda"))
    per_row = {n: torch.ones(2, device="cuda") for n in ("repetition", "frequency", "presence")}
    return [
        (K.ckks_clear_layer_norm, dict(x=x, weight=w, bias=b, out=torch.empty_like(x)), ("x", "weight", "bias", "out"), ("out",)),
        (K.ckks_clear_layer_norm_grad, dict(dy=dy, x=x, mean=mean, rstd=rstd, weight=w, dx=torch.empty_like(x)), ("dy", "x", "mean", "rstd", "weight", "dx"), ("dx",)),
        (K.ckks_clear_cache_append, dict(new, **page, q=c.q, q_out=torch.empty_like(c.q), cos=torch.ones(32, 32, device="cuda"), sin=torch.ones(32, 32, device="cuda")),
         ("k", "v", "k_pages", "v_pages", "q", "q_out", "cos", "sin"), ("k_pages", "v_pages", "q_out")),
        (K.ckks_clear_cache_append, dict(new, **page), ("k", "k_pages"), ("k_pages", "v_pages")),
        (K.ckks_clear_attend, dict(page, q=c.q, out=torch.empty_like(c.q), lse=torch.empty(4, 4, device="cuda")), ("q", "k_pages", "v_pages", "out", "lse"), ("out", "lse")),
        (K.ckks_clear_logits, dict(words, **per_row, logits=randn(g, 2, 50), bias=torch.ones(1, device="cuda"), out=torch.empty(2, 50, device="cuda")),
         ("logits", "repetition", "frequency", "presence", "bias", "out"), ("out",)),
    ]


def test_tensors_that_require_a_gradient_are_refused():
    from paper_2604_09975_amd import clear as K
    for call, args, floats, _ in calls(K):
        for name in floats:
            t = dict(args, **{name: args[name].detach().clone().requires_grad_()})
            with pytest.raises(ValueError, match="requires a gradient"):
                call(**t)
            with torch.no_grad():
                got = call(**t)
            assert not any(o.grad_fn is not None for o in (got if isinstance(got, tuple) else (got,)) if o is not None)
        # computed from one that does
        t = dict(args, **{floats[0]: args[floats[0]].detach().clone().requires_grad_() * 1})
        with pytest.raises(ValueError, match="requires a gradient"):
            call(**t)
        call(**args)


def test_what_is_written_in_place_counts_as_modified():
    from paper_2604_09975_amd import clear as K
    for call, args, _, written in calls(K):
        before = {n: t._version for n, t in args.items()}
        call(**args)
        assert {n for n, t in args.items() if t._version != before[n]} == set(written)
    # so a backward pass that needs the old values does not take the new ones
    x, w = randn(gen(2), 4, 64), torch.ones(64, device="cuda", requires_grad=True)
    loss = (x * w).sum()
    K.ckks_clear_layer_norm(x, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_inference_mode():
    from paper_2604_09975_amd import clear as K
    with torch.inference_mode():
        for call, args, _, _ in calls(K):
            call(**args)
