"""A small pruned decoder that answers with drafted tokens: everything a step needs, on this library.

Per layer: q, k and v as products with bias, keys and values written into a paged cache (8 bits), attention of the new tokens over it,
the output projection with bias and residual, the MLP with bias and ReLU and with bias and residual; at the end the check of the drafts.
The drafts are what followed the last tokens when they last occurred; random weights, so what is said means nothing.  Activations are
columns, (hidden, nb) with nb in {1, 2, 4, 8}, as the products take and leave them; PyTorch does the norms and the softmax.

    python examples/drafted_decoding.py [--drafts 7] [--tokens 48] [--bits 8] [--sample]
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2507_12205_amd as E                        # noqa: E402
from paper_2507_12205_amd import device as D            # noqa: E402

HIDDEN, HEADS, KV_HEADS, DIM, MLP, VOCAB, LAYERS, PAGE, PAGES = 256, 4, 2, 64, 512, 512, 2, 16, 64


class Linear:
    """A pruned matrix as an EC-CSR image on the device, and its bias."""

    def __init__(self, rng, m, n, gain=1.0):
        w = np.where(rng.random((m, n)) < 0.4, rng.normal(size=(m, n)) * gain / math.sqrt(0.4 * n), 0).astype(np.float16)
        self.m, self.dense = m, torch.from_numpy(w)
        self.image = E.ecspmv_build_dense(w, E.make_opts(delta_bits=4))
        D.upload(self.image)
        self.bias = torch.from_numpy((0.1 * rng.normal(size=m)).astype(np.float16)).cuda()

    def __call__(self, x, activation="none", residual=None):
        y = torch.empty((self.m, x.shape[1]), dtype=torch.float16, device="cuda")
        return D.run_epilogue(self.image, x, y, self.bias, activation, None, residual)


class Decoder:
    def __init__(self, seed=0, bits=8):
        rng = np.random.default_rng(seed)
        self.embed = torch.from_numpy(rng.normal(size=(VOCAB, HIDDEN)).astype(np.float16)).cuda()
        self.position = torch.from_numpy((0.5 * rng.normal(size=(PAGES * PAGE, HIDDEN))).astype(np.float16)).cuda()
        self.layers = [dict(q=Linear(rng, HEADS * DIM, HIDDEN), k=Linear(rng, KV_HEADS * DIM, HIDDEN), v=Linear(rng, KV_HEADS * DIM, HIDDEN),
                            o=Linear(rng, HIDDEN, HEADS * DIM), up=Linear(rng, MLP, HIDDEN), down=Linear(rng, HIDDEN, MLP))
                       for _ in range(LAYERS)]
        self.head = Linear(rng, VOCAB, HIDDEN, gain=3.0)
        self.caches = [D.kv_cache(PAGES, KV_HEADS, PAGE, DIM, bits) for _ in range(LAYERS)]
        pages = rng.permutation(PAGES).astype(np.int32)                 # one sequence, pages in no order
        self.table = torch.from_numpy(pages[None]).cuda()
        self.slots = (self.table[0].long()[:, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten()

    @staticmethod
    def norm(x):
        return torch.nn.functional.layer_norm(x.t().float(), (HIDDEN,)).t().half().contiguous()

    def logits(self, tokens, past):
        """Logits (len(tokens), VOCAB) FP32 after each of up to eight new tokens that follow `past` others."""
        new = len(tokens)
        nb = next(n for n in (1, 2, 4, 8) if n >= new)                  # the columns beyond the new tokens are zeros
        x = torch.zeros((HIDDEN, nb), dtype=torch.float16, device="cuda")
        x[:, :new] = (self.embed[torch.tensor(tokens, device="cuda")] + self.position[past:past + new]).t()
        slots = torch.full((nb,), -1, dtype=torch.int64, device="cuda")
        slots[:new] = self.slots[past:past + new]
        start = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        total = torch.tensor([past + new], dtype=torch.int32, device="cuda")

        def heads(y, count):                                            # (count * DIM, nb) as (token, head, value): a view
            return y.view(count, DIM, nb).permute(2, 0, 1)
        for layer, cache in zip(self.layers, self.caches):
            h = self.norm(x)
            q, k, v = (layer[name](h) for name in "qkv")
            D.kv_write(cache, heads(k, KV_HEADS), heads(v, KV_HEADS), slots)
            a = torch.zeros_like(q)
            D.attention(cache, heads(q, HEADS), heads(a, HEADS), start, total, self.table, new)
            x = layer["o"](a, residual=x)
            x = layer["down"](layer["up"](self.norm(x), "relu"), residual=x)
        return self.head(self.norm(x)).t()[:new].float()


def drafts_for(tokens, most):
    """What followed when the last two tokens (or else the last one) were last seen."""
    for n in (2, 1):
        for i in range(len(tokens) - n - 1, -1, -1):
            if tokens[i:i + n] == tokens[-n:]:
                return tokens[i + n:i + n + most]
    return []


def generate(model, prompt, count, drafts=7, sample=False, seed=0):
    """`count` tokens after the prompt, and in how many steps.  Without `sample` the likeliest token every time."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    tokens, past, steps = list(prompt), 0, 0
    while past + 8 < len(tokens):                                       # the prompt, eight tokens at a time
        model.logits(tokens[past:past + 8], past)
        past += 8
    while len(tokens) < len(prompt) + count:
        waiting = tokens[past:]                                         # not yet in the cache
        guess = drafts_for(tokens, min(drafts, 8 - len(waiting), len(prompt) + count - len(tokens) - 1))
        logits = model.logits(waiting + guess, past)[len(waiting) - 1:]
        target = torch.softmax(logits, -1)
        if not sample:
            target = torch.nn.functional.one_hot(target.argmax(-1), VOCAB).float()
        drafted = torch.tensor([guess], dtype=torch.int32, device="cuda").view(1, len(guess))
        uniform = torch.rand((1, len(guess) + 1), generator=g, device="cuda")
        out = torch.empty((1, len(guess) + 1), dtype=torch.int32, device="cuda")
        accepted = torch.empty(1, dtype=torch.int32, device="cuda")
        D.verify(target[None], None, drafted, uniform, out, accepted)
        n = int(accepted)
        past = len(tokens) + n                                          # refused drafts are overwritten by what comes
        tokens += out[0, :n + 1].tolist()
        steps += 1
    return tokens[len(prompt):], steps


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--drafts", type=int, default=7)
    p.add_argument("--tokens", type=int, default=48)
    p.add_argument("--bits", type=int, default=8)
    p.add_argument("--sample", action="store_true")
    a = p.parse_args()
    model = Decoder(bits=a.bits)
    prompt = [int(t) for t in np.random.default_rng(1).integers(0, VOCAB, 6)] * 3
    tokens, steps = generate(model, prompt, a.tokens, a.drafts, a.sample)
    print("prompt", prompt)
    print("tokens", tokens)
    print(f"{len(tokens)} tokens in {steps} steps")


if __name__ == "__main__":
    main()
