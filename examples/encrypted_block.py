"""Text from a small block whose projections run on ciphertexts: `python examples/encrypted_block.py` on an MI355X.

The server holds the plaintext weights of the QKV and the output projection and sees ciphertexts only.  The key holder decrypts
between the two and does the rest in the clear on the same device: layer norm, the paged key / value cache with the position
rotation, attention of a chunk of tokens over it, and the rules on the logits.  A prompt goes through in chunks of one segment,
the new tokens one at a time through the same calls.  With `packed` the cache takes a byte for each entry, and with `draw` the next token
is drawn instead of taken as the largest.  `tune` trains the parameters of the last layer norm, which the key holder
can do alone: they meet no ciphertext.

Random weights; a ring of 2^13 (three 45-bit primes, one special prime), so that it runs in seconds.
"""
import math
import os
import sys

import numpy as np
import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_09975_amd import binding as B
from paper_2604_09975_amd import clear as K
from paper_2604_09975_amd import client as CL

SEGMENT, WIDTH, HEADS, KV_HEADS, DIM, VOCAB, PAGE = 16, 64, 4, 2, 16, 200, 8
COLUMNS, BABY, LEVEL, SCALE = 64, 8, 3, 2.0**35


class Projection:
    """Y = XW on ciphertexts: the key holder's encrypt and decrypt around the server's ckks_ctpt_matmul."""

    def __init__(self, P, client, keys, weight):
        self.P, self.client, self.keys, self.n = P, client, keys, P.N // 2
        d_in, self.d_out = weight.shape
        groups, self.blocks, giants = -(-d_in // COLUMNS), -(-self.d_out // COLUMNS), COLUMNS // BABY
        self.weights = B.ckks_weights_create(P, LEVEL, SEGMENT, COLUMNS, groups, self.blocks, BABY)
        for b in range(self.blocks):
            for p in range(giants):
                z = CL.diagonal_slots(weight, SEGMENT, self.n, COLUMNS, BABY, b, p).reshape(groups * BABY, self.n)
                B.ckks_weights_set_diagonals(self.weights, (b * giants + p) * groups * BABY, client.enc.encode(z, SCALE))

    def __call__(self, x):
        """x: float32 device tensor of up to SEGMENT rows -> float32 device tensor [rows][d_out]."""
        rows = np.zeros((SEGMENT, x.shape[1]))
        rows[:x.shape[0]] = x.double().cpu().numpy()
        ct = torch.stack([self.client.encrypt_slots(z, SCALE, LEVEL) for z in CL.pack_columns(rows, self.n, COLUMNS)])
        y, _ = B.ckks_ctpt_matmul(self.P, self.weights, ct, *self.keys, flags=B.MATMUL_MERGED_GIANT | B.MATMUL_RESCALE)
        scale = SCALE * SCALE / self.P.q[LEVEL - 1]
        slots = np.stack([self.client.decrypt_slots(y[b], LEVEL - 1, scale) for b in range(self.blocks)])
        out = CL.unpack_columns(slots.real, SEGMENT, COLUMNS, self.d_out)[:x.shape[0]]
        return torch.from_numpy(np.ascontiguousarray(out, dtype=np.float32)).cuda()


class Block:
    """Embedding, layer norm, attention, residual, layer norm, logits.  packed: float8_e4m3fn or int8 for a cache of 8 bits."""

    def __init__(self, seed=1, max_tokens=96, packed=None):
        r = np.random.default_rng(seed)
        P = B.ckks_params_create(13, B.ckks_find_primes(45, 13, 3), B.ckks_find_primes(50, 13, 1), 3)
        client = CL.Client(P, seed)
        keys = ([client.galois_key(q * SEGMENT) for q in range(1, BABY)],
                [client.galois_key(p * BABY * SEGMENT) for p in range(1, COLUMNS // BABY)])
        self.w_qkv = r.normal(0, 1.5 / math.sqrt(WIDTH), (WIDTH, (HEADS + 2 * KV_HEADS) * DIM))
        self.w_out = r.normal(0, 1 / math.sqrt(HEADS * DIM), (HEADS * DIM, WIDTH))
        self.qkv, self.out = Projection(P, client, keys, self.w_qkv), Projection(P, client, keys, self.w_out)

        def device(a):
            return torch.from_numpy(a.astype(np.float32)).cuda()
        self.embedding = device(r.normal(0, 1, (VOCAB, WIDTH)))
        self.head = device(r.normal(0, 1 / math.sqrt(WIDTH), (WIDTH, VOCAB)))
        self.norms = [(device(1 + 0.1 * r.normal(size=WIDTH)), device(0.1 * r.normal(size=WIDTH))) for _ in range(2)]
        # one conversation's cache: its pages need not lie in order
        pages = -(-max_tokens // PAGE)
        self.cache = [torch.zeros(pages, KV_HEADS, PAGE, DIM, device="cuda", dtype=packed or torch.float32) for _ in range(2)]
        if packed:  # and a power of two for each 32 entries of a head
            self.cache += [torch.zeros(pages, KV_HEADS, PAGE, -(-DIM // 32), device="cuda", dtype=torch.uint8) for _ in range(2)]
        self.append, self.attend = ((K.ckks_clear_packed_append, K.ckks_clear_packed_attend) if packed else
                                    (K.ckks_clear_cache_append, K.ckks_clear_attend))
        self.page_table = torch.from_numpy(r.permutation(pages).astype(np.int32)[None]).cuda()
        angle = np.arange(pages * PAGE)[:, None] * 10000.0 ** (-np.arange(0, DIM, 2) / DIM)
        self.cos, self.sin = device(np.cos(angle)), device(np.sin(angle))
        self.length = 0

    def chunk(self, tokens):
        """Up to SEGMENT tokens through the block: the rows before the last layer norm."""
        n = len(tokens)
        if self.length + n > self.page_table.shape[1] * PAGE:
            raise ValueError(f"{self.length + n} tokens in a cache of {self.page_table.shape[1] * PAGE}")
        self.length += n
        batch = (self.page_table, torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                 torch.tensor([self.length], dtype=torch.int32, device="cuda"))
        x = self.embedding[torch.tensor(tokens, device="cuda")]
        h, _, _ = K.ckks_clear_layer_norm(x, *self.norms[0])
        qkv = self.qkv(h)
        q, k, v = qkv.view(n, HEADS + 2 * KV_HEADS, DIM).split((HEADS, KV_HEADS, KV_HEADS), dim=1)
        q = self.append(k, v, *self.cache, *batch, cos=self.cos, sin=self.sin, q=q)
        a = self.attend(q, *self.cache, *batch)
        return x + self.out(a.view(n, HEADS * DIM))

    def generate(self, prompt, count, allowed=None, draw=None):
        """-> (tokens, the rows before the last layer norm, the logits under the rules, step by step).  draw: `count` numbers of [0, 1) by
        which tokens are drawn (of the 20 likeliest, those that make up 0.9)."""
        tokens, rows, steps = list(prompt), [], []
        start = torch.empty(2, dtype=torch.int32, device="cuda")
        mask = None
        if allowed is not None:  # a grammar that admits these words only
            bits = np.zeros((VOCAB + 31) // 32 * 32, dtype=np.uint32)
            bits[list(allowed)] = 1
            mask = torch.from_numpy((bits.reshape(-1, 32) << np.arange(32, dtype=np.uint32)).sum(1, dtype=np.uint32).view(np.int32)).cuda()[None]
        todo = list(prompt)
        while len(tokens) < len(prompt) + count:
            while todo:
                rows.append(self.chunk(todo[:SEGMENT]))
                todo = todo[SEGMENT:]
            y, _, _ = K.ckks_clear_layer_norm(rows[-1][-1:], *self.norms[1])
            logits = y @ self.head
            start.copy_(torch.tensor([0, len(tokens)], dtype=torch.int32))
            logits = K.ckks_clear_logits(
                logits, out=logits, tokens=torch.tensor(tokens, dtype=torch.int32, device="cuda"), token_start=start,
                n_prompt=torch.tensor([len(prompt)], dtype=torch.int32, device="cuda"), repetition=torch.full((1,), 1.3, device="cuda"),
                presence=torch.full((1,), 0.5, device="cuda"), bias_ids=torch.tensor([7], dtype=torch.int32, device="cuda"),
                bias=torch.full((1,), 2.0, device="cuda"), bias_start=torch.tensor([0, 1], dtype=torch.int32, device="cuda"), mask=mask)
            steps.append(logits[0].clone())
            if draw is None:
                tokens.append(int(logits.argmax()))
            else:
                tokens.append(int(K.ckks_clear_sample(logits, torch.full((1,), float(draw[len(tokens) - len(prompt)]), device="cuda"),
                                                      top_k=torch.full((1,), 20, dtype=torch.int32, device="cuda"), top_p=torch.full((1,), 0.9, device="cuda"))))
            todo = tokens[-1:]
        return tokens, torch.cat(rows), steps

    def tune(self, rows, target, rate, count):
        """Gradient steps on the last layer norm's weight and bias towards `target` -> the mean squared error before each."""
        weight, bias = self.norms[1]
        errors = []
        for _ in range(count):
            y, mean, rstd = K.ckks_clear_layer_norm(rows, weight, bias)
            off = y - target
            errors.append(float((off * off).mean()))
            _, dw, db = K.ckks_clear_layer_norm_grad(off.mul_(2 / off.numel()), rows, mean, rstd, weight)
            weight -= rate * dw
            bias -= rate * db
        return errors


def main():
    block = Block()
    prompt = np.random.default_rng(2).integers(0, VOCAB, 37).tolist()
    tokens, rows, _ = block.generate(prompt, 8, allowed=range(0, VOCAB, 2))
    print("prompt  ", *prompt)
    print("answer  ", *tokens[len(prompt):])
    small = Block(packed=torch.int8)
    drawn, _, _ = small.generate(prompt, 8, allowed=range(0, VOCAB, 2), draw=np.random.default_rng(3).random(8))
    print("drawn   ", *drawn[len(prompt):])
    # what another weight and bias would have given
    target, _, _ = K.ckks_clear_layer_norm(rows, block.norms[0][0] * 1.5, block.norms[0][1] + 0.5)
    errors = block.tune(rows, target, 20.0, 20)
    print(f"last layer norm tuned: mean squared error {errors[0]:.2e} -> {errors[-1]:.2e}")


if __name__ == "__main__":
    main()
