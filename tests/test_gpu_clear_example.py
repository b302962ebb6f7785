"""The example that runs the steps in the clear between encrypted projections, against the same block in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def plain(block, tokens, prompt, allowed):
    """Rows before the last layer norm and the logits under the rules after every token from the prompt's last on."""
    from examples import encrypted_block as X

    def norm(x, wb):
        w, b = (t.double().cpu().numpy() for t in wb)
        d = x - x.mean(-1, keepdims=True)
        return d / np.sqrt((d * d).mean(-1, keepdims=True) + 1e-5) * w + b
    emb = block.embedding.double().cpu().numpy()
    x = emb[tokens]
    n = len(tokens)
    qkv = (norm(x, block.norms[0]) @ block.w_qkv).reshape(n, -1, X.DIM)
    half = X.DIM // 2
    angle = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, X.DIM, 2) / X.DIM)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = qkv[..., :half], qkv[..., half:]
    turned = np.concatenate((a * c - b * s, b * c + a * s), -1)
    out = np.zeros((n, X.HEADS, X.DIM))
    for h in range(X.HEADS):
        k, v = turned[:, X.HEADS + h * X.KV_HEADS // X.HEADS], qkv[:, X.HEADS + X.KV_HEADS + h * X.KV_HEADS // X.HEADS]
        z = turned[:, h] @ k.T / np.sqrt(X.DIM)
        z[np.triu_indices(n, 1)] = -np.inf
        p = np.exp(z - z.max(-1, keepdims=True))
        out[:, h] = p / p.sum(-1, keepdims=True) @ v
    rows = x + out.reshape(n, -1) @ block.w_out
    steps = []
    for t in range(len(prompt) - 1, n):
        l = norm(rows[t], block.norms[1]) @ block.head.double().cpu().numpy()
        past = tokens[:t + 1]
        for w in set(past):
            l[w] = l[w] / 1.3 if l[w] > 0 else l[w] * 1.3
        for w in set(past[len(prompt):]):
            l[w] -= 0.5
        l[7] += 2
        l[[w for w in range(X.VOCAB) if w not in allowed]] = -np.inf
        steps.append(l)
    return rows, steps


def test_generation_and_tuning():
    from examples import encrypted_block as X
    block = X.Block(seed=4, max_tokens=64)
    prompt = np.random.default_rng(5).integers(0, X.VOCAB, 37).tolist()
    allowed = set(range(0, X.VOCAB, 3)) | {7}
    tokens, rows, steps = block.generate(prompt, 6, allowed)
    assert len(tokens) == 43 and all(t in allowed for t in tokens[37:])
    want, logits = plain(block, tokens[:-1], prompt, allowed)
    # two projections whose slots are off by up to 1e-3 each (the bound of the decrypted values): the output's entries sum 64 of
    # the first's by weights of size 1/8, attention and norms of deviation 1 add no more than that again
    assert np.abs(rows.cpu().numpy() - want).max() < 2e-2
    for got, l in zip(steps, logits):
        got = got.double().cpu().numpy()
        assert (np.isinf(got) == np.isinf(l)).all()
        keep = np.isfinite(l)
        # a logit is a product of 64 entries, each off by 2e-2 / deviation at most, with entries of size 1/8
        assert np.abs(got[keep] - l[keep]).max() < 0.3
        order = np.sort(l[keep])
        if order[-1] - order[-2] > 0.6:
            assert got.argmax() == l.argmax()
    from paper_2604_09975_amd import clear as K
    target, _, _ = K.ckks_clear_layer_norm(rows, block.norms[0][0] * 1.5, block.norms[0][1] + 0.5)
    # the loss is quadratic in both parameters with second derivatives of about 2 / 64 x (1 + off-diagonal parts of a few tenths):
    # a rate of 20 leaves less than 0.8 of the distance a step
    errors = block.tune(rows, target, 20.0, 30)
    assert errors[-1] < 1e-3 * errors[0] and all(b <= a for a, b in zip(errors, errors[1:]))
