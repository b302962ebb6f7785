"""Rules on more rows of logits than one launch has threads for: each row as it comes out of a call of fewer."""
import pytest
import torch

from tests.clear_util import gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rules", [False, True])
def test_rows(rules):
    from paper_2604_09975_amd import clear as K
    rows, vocab = (1 << 22) + 77, 24
    g = gen(1)
    logits = randn(g, rows, vocab, dtype=torch.bfloat16)
    mask = torch.randint(-2**31, 2**31 - 1, (rows, 1), generator=g, device="cuda").to(torch.int32)
    per_row = {}
    if rules:
        tokens = torch.randint(0, vocab, (2 * rows,), generator=g, device="cuda", dtype=torch.int32)
        start = torch.arange(0, 2 * rows + 1, 2, dtype=torch.int32, device="cuda")
        ids = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
        bias, bias_start = randn(g, rows), torch.arange(rows + 1, dtype=torch.int32, device="cuda")
        per_row = {"n_prompt": torch.ones(rows, dtype=torch.int32, device="cuda"), "repetition": 1 + torch.rand(rows, generator=g, device="cuda"),
                   "frequency": torch.rand(rows, generator=g, device="cuda"), "presence": torch.rand(rows, generator=g, device="cuda")}
    out = torch.full((rows, vocab), 7.0, device="cuda")

    def call(at, end, out):
        more = {k: x[at:end] for k, x in per_row.items()}
        if rules:
            more.update(tokens=tokens, token_start=start[at:end + 1], bias_ids=ids, bias=bias, bias_start=bias_start[at:end + 1])
        return K.ckks_clear_logits(logits[at:end], out=out, mask=mask[at:end], **more)
    call(0, rows, out)
    for at in (0, (1 << 21) - 500, (1 << 21) - 1, (1 << 22) - 999, rows - 1000):
        assert torch.equal(call(at, at + 1000, torch.empty(1000, vocab, device="cuda")), out[at:at + 1000])
    assert int((out == 7.0).sum()) < rows // 1000
