"""A small pruned decoder that answers with trees of drafted tokens: positions by rotation, every node of a tree in one pass, the accepted path kept.

A step's new tokens are the one that waits and up to seven nodes below it.  Per layer: q, k and v as products with bias, keys rotated by their
tokens' positions (a node's depth) and written into a paged cache with the values, queries rotated in place; attention in which a node sees its own
path and what came before; the rest as in drafted_decoding.py.  At the end the check of the tree, and the accepted path's rows are moved in all layers'
caches to where they follow one another.  The nodes are what followed the last tokens each time they occurred before; random weights, so what is
said means nothing.

    python examples/drafted_tree.py [--nodes 7] [--tokens 48] [--bits 8] [--sample]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from drafted_decoding import DIM, HEADS, HIDDEN, KV_HEADS, VOCAB, D, Decoder    # noqa: E402


class TreeDecoder(Decoder):
    """Positions are angles of q and k, and not added to the tokens."""

    def __init__(self, seed=0, bits=8):
        super().__init__(seed, bits)
        self.frequency = D.rotary_frequency(DIM // 2)
        self.all_caches = D.KvCaches(self.caches)

    def logits(self, tokens, past, parents=None):
        """Logits (len(tokens), VOCAB) FP32 after each of up to eight new tokens that follow `past` others.  parents: the number of each token's
        parent among them, -1 for the first (None: each follows the one before it)."""
        new = len(tokens)
        parents = list(range(-1, new - 1)) if parents is None else parents
        depth = []
        for p in parents:
            depth.append(depth[p] + 1 if p >= 0 else 0)
        nb = next(n for n in (1, 2, 4, 8) if n >= new)                  # the columns beyond the new tokens are zeros
        x = torch.zeros((HIDDEN, nb), dtype=torch.float16, device="cuda")
        x[:, :new] = self.embed[torch.tensor(tokens, device="cuda")].t()
        slots = torch.full((nb,), -1, dtype=torch.int64, device="cuda")
        slots[:new] = self.slots[past:past + new]
        position = torch.zeros(nb, dtype=torch.int32, device="cuda")
        position[:new] = past + torch.tensor(depth, dtype=torch.int32, device="cuda")
        start = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        total = torch.tensor([past + new], dtype=torch.int32, device="cuda")
        seen = torch.zeros((nb, 1), dtype=torch.int32, device="cuda")
        seen[:new] = D.tree_seen([parents])

        def heads(y, count):                                            # (count * DIM, nb) as (token, head, value): a view
            return y.view(count, DIM, nb).permute(2, 0, 1)
        for layer, cache in zip(self.layers, self.caches):
            h = self.norm(x)
            q, k, v = (layer[name](h) for name in "qkv")
            D.kv_append(cache, heads(k, KV_HEADS), heads(v, KV_HEADS), slots, position, self.frequency, heads(q, HEADS))
            a = torch.zeros_like(q)
            D.attention_tree(cache, heads(q, HEADS), heads(a, HEADS), start, total, self.table, seen, new)
            x = layer["o"](a, residual=x)
            x = layer["down"](layer["up"](self.norm(x), "relu"), residual=x)
        return self.head(self.norm(x)).t()[:new].float()

    def keep(self, past, path, accepted):
        """The accepted nodes' rows behind the `past` tokens and the one that waited."""
        D.kv_keep(self.all_caches, torch.tensor([past + 1], dtype=torch.int32, device="cuda"), path, accepted, self.table)


def tree_for(tokens, most):
    """(tokens, parents) of up to `most` nodes: what followed each time that the last two tokens (or else the last one) were seen, the latest first,
    with common beginnings in common."""
    drafted, parent = [], []
    for n in (2, 1):
        for i in range(len(tokens) - n - 1, -1, -1):
            if tokens[i:i + n] != tokens[-n:]:
                continue
            at = -1
            for x in tokens[i + n:i + n + 4]:
                same = [j for j in range(len(drafted)) if parent[j] == at and drafted[j] == x]
                if not same and len(drafted) == most:
                    break
                if not same:
                    drafted.append(x)
                    parent.append(at)
                at = same[0] if same else len(drafted) - 1
    return drafted, parent


def generate(model, prompt, count, nodes=7, sample=False, seed=0):
    """`count` tokens after the prompt, and in how many steps.  Without `sample` the likeliest token every time."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    tokens, past, steps = list(prompt), 0, 0
    while past < len(tokens) - 1:                                       # the prompt but for its last token, eight at a time
        chunk = tokens[past:min(past + 8, len(tokens) - 1)]
        model.logits(chunk, past)
        past += len(chunk)
    while len(tokens) < len(prompt) + count:
        guess, parent = tree_for(tokens, min(nodes, 7))
        target = torch.softmax(model.logits(tokens[past:] + guess, past, [-1] + [p + 1 for p in parent]), -1)
        if not sample:
            target = torch.nn.functional.one_hot(target.argmax(-1), VOCAB).float()
        made = len(guess)
        drafted, below = (torch.tensor([x], dtype=torch.int32, device="cuda").view(1, made) for x in (guess, parent))
        uniform = torch.rand((1, made + 1), generator=g, device="cuda")
        out, path, accepted = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((1, made + 1), (1, made), (1,)))
        D.verify_tree(target[None], drafted, below, uniform, out, path, accepted)
        model.keep(past, path, accepted)
        n = int(accepted)
        past += 1 + n                                                   # refused nodes are overwritten by what comes
        tokens += out[0, :n + 1].tolist()
        steps += 1
    return tokens[len(prompt):len(prompt) + count], steps


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--nodes", type=int, default=7)
    p.add_argument("--tokens", type=int, default=48)
    p.add_argument("--bits", type=int, default=8)
    p.add_argument("--sample", action="store_true")
    a = p.parse_args()
    model = TreeDecoder(bits=a.bits)
    prompt = [int(t) for t in np.random.default_rng(1).integers(0, VOCAB, 6)] * 3
    tokens, steps = generate(model, prompt, a.tokens, a.nodes, a.sample)
    print("prompt", prompt)
    print("tokens", tokens)
    print(f"{len(tokens)} tokens in {steps} steps")


if __name__ == "__main__":
    main()
