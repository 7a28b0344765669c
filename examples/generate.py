"""A small network of AAP layers that writes sequences of tokens, served with a paged int8 cache.

Each block is an attention and a feed-forward layer, every product one of int8 codes with 2-bit weights:

  h       = h + Quant(attend(q)) Wo^T                       q, k, v = Quant(norm(h)) Wqkv^T; k and v into the cache
  h       = h + Quant(norm(relu(Quant(norm(h)) W1^T))) W2^T
  logits  = Quant(norm(h)) Whead^T, and the next token by `sample`

A prompt is taken in one token at a time here, like the tokens after it: kv_append writes a token's keys and values,
paged_attention reads those of its sequence.  Sequences of different lengths run side by side; one that is over leaves its
place in the batch free (length 0).

    python examples/generate.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2410_05911_gb300 import aecct  # noqa: E402


class Model:
    """Random weights of a trained model's shapes: d wide, `heads` query heads over `kv_heads` of keys and values."""

    def __init__(self, vocab=1000, d=128, layers=2, heads=8, kv_heads=2, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.d, self.heads, self.kv_heads, self.dim, self.dtype = vocab, d, heads, kv_heads, d // heads, dtype

        def ternary(n, k):
            (t,), scale, _ = aecct.aap_ternarize([torch.randn((n, k), device="cuda", generator=g) * k ** -0.5])
            return t, scale

        wide = (heads + 2 * kv_heads) * self.dim
        self.blocks = [dict(qkv=ternary(wide, d), o=ternary(d, d), up=ternary(4 * d, d), down=ternary(d, 4 * d),
                            g1=torch.ones(d, device="cuda"), g2=torch.ones(d, device="cuda"), g3=torch.ones(d, device="cuda"),
                            g4=torch.ones(4 * d, device="cuda")) for _ in range(layers)]
        self.embedding = torch.randn((vocab, d), device="cuda", generator=g).to(dtype)
        self.head, self.g = ternary(vocab, d), torch.ones(d, device="cuda")

    def caches(self, pages, page_size):
        return [aecct.kv_cache(pages, self.kv_heads, page_size, self.dim) for _ in self.blocks]

    def _linear(self, x, gain, weights):
        codes, scale, _, _ = aecct.rms_quant(x, gain)
        return aecct.aap_linear(codes, scale, *weights, dtype=self.dtype)

    def step(self, tokens, caches, table, lengths):
        """Logits for the token after `tokens` [batch], the newest of sequences of `lengths` tokens."""
        h = self.embedding[tokens]
        for block, cache in zip(self.blocks, caches):
            qkv = self._linear(h, block["g1"], block["qkv"]).view(len(tokens), -1, self.dim)
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
            aecct.kv_append(k, v, cache, table, lengths)
            out, _ = aecct.paged_attention(q, cache, table, lengths)
            h = h + self._linear(out.reshape(len(tokens), self.d), block["g2"], block["o"])
            h = h + self._linear(torch.relu(self._linear(h, block["g3"], block["up"])), block["g4"], block["down"])
        return self._linear(h, self.g, self.head)


def generate(model, prompts, new, page_size=16, temperature=0.8, top_k=50, top_p=0.95, seed=0):
    """`new` tokens after each of `prompts` (lists of tokens).  Returns the sequences."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    batch, longest = len(prompts), max(len(p) for p in prompts) + new
    columns = -(-longest // page_size)
    table = torch.randperm(batch * columns, device="cuda", generator=g).int().view(batch, columns)  # each sequence's pages, anywhere
    caches = model.caches(batch * columns, page_size)
    sequences = [list(p) for p in prompts]
    for at in range(longest - 1):
        over = [at + 1 >= len(p) + new for p in prompts]
        tokens = torch.tensor([s[min(at, len(s) - 1)] for s in sequences], device="cuda")
        lengths = torch.tensor([0 if o else at + 1 for o in over], dtype=torch.int32, device="cuda")
        logits = model.step(tokens, caches, table, lengths)
        u = torch.rand((batch,), device="cuda", generator=g)
        picked = aecct.sample(logits, u, temperature=temperature, top_k=top_k, top_p=top_p).tolist()
        for s, token, o in zip(sequences, picked, over):
            if at + 1 == len(s) and not o:
                s.append(token)
    return sequences


def main() -> None:
    model = Model()
    prompts = [[1, 2, 3], [5], [7, 8, 9, 10, 11]]
    for prompt, s in zip(prompts, generate(model, prompts, new=20)):
        print(prompt, "->", s[len(prompt):])


if __name__ == "__main__":
    main()
