"""The example that runs rotation, attention of trees, their check and the keeping of accepted paths together: with trees it says what it says
without, a node's logits are those of its path as a row, and all of them those of the same decoder in dense 64-bit arithmetic."""
import math
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_trees_change_nothing(bits):
    import drafted_tree as X
    prompt = [int(t) for t in np.random.default_rng(3).integers(0, X.VOCAB, 5)] * 3
    plain, steps = X.generate(X.TreeDecoder(bits=bits), prompt, 30, nodes=0)
    assert steps == 30 and len(plain) == 30
    # the answer as part of what is drafted from: many nodes are accepted, and their rows moved
    draft = X.tree_for
    try:
        X.tree_for = lambda tokens, most: follow(prompt + plain, tokens, most, np.random.default_rng(len(tokens)))
        drafted, fewer = X.generate(X.TreeDecoder(bits=bits), prompt, 30, nodes=7)
    finally:
        X.tree_for = draft
    assert drafted == plain and fewer < 20
    again, _ = X.generate(X.TreeDecoder(bits=bits), prompt, 30, nodes=7)
    assert again == plain
    sampled, _ = X.generate(X.TreeDecoder(bits=bits), prompt, 30, nodes=7, sample=True)
    assert len(sampled) == 30 and all(0 <= t < X.VOCAB for t in sampled)


def follow(answer, tokens, most, rng):
    """A tree with the next three tokens of the answer in it, behind and among nodes that are wrong."""
    right, drafted, parent, at = answer[len(tokens):len(tokens) + 3], [], [], -1
    for x in right:
        for _ in range(int(rng.integers(0, 2))):
            drafted.append(int((x + rng.integers(1, 9)) % 512))
            parent.append(at)
        drafted.append(x)
        parent.append(at)
        at = len(drafted) - 1
    return drafted[:most], parent[:most]


def dense_logits(X, model, tokens, position, seen):
    import torch
    x = model.embed[torch.tensor(tokens)].double().cpu()
    n, pairs = len(tokens), X.DIM // 2
    angle = torch.tensor(position, dtype=torch.float64)[:, None] * model.frequency.cpu()
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

    def lin(m, v):
        return v @ m.dense.double().t() + m.bias.double().cpu()

    def norm(v):
        return torch.nn.functional.layer_norm(v, (X.HIDDEN,))

    def turn(v):
        a, b = v[..., :pairs], v[..., pairs:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    mask = torch.where(torch.tensor(seen), 0.0, -math.inf).double()
    for layer in model.layers:
        h = norm(x)
        q, k = turn(lin(layer["q"], h).view(n, -1, X.DIM)), turn(lin(layer["k"], h).view(n, -1, X.DIM))
        v = lin(layer["v"], h).view(n, -1, X.DIM)
        k, v = (t.repeat_interleave(X.HEADS // X.KV_HEADS, 1) for t in (k, v))
        s = torch.softmax(torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(X.DIM) + mask, -1)
        x = x + lin(layer["o"], torch.einsum("hij,jhd->ihd", s, v).reshape(n, -1))
        x = x + lin(layer["down"], torch.relu(lin(layer["up"], norm(x))))
    return lin(model.head, norm(x))


def test_logits_of_a_tree_against_dense_64_bits():
    """FP16 activations between the operators: every layer rounds some ten times at 2^-11, on values of about 1; a tenth of that in sum."""
    import torch
    import drafted_tree as X
    model, rng = X.TreeDecoder(bits=16), np.random.default_rng(4)
    tokens = [int(t) for t in rng.integers(0, X.VOCAB, 27)]
    parents = [-1, 0, 1, 0, 3, 3, 2, 4]
    depth = [0, 1, 2, 1, 2, 2, 3, 3]
    got = [model.logits(tokens[i:i + 8], i) for i in (0, 8)] + [model.logits(tokens[16:19], 16)] + [model.logits(tokens[19:27], 19, parents)]
    seen = np.tril(np.ones((27, 27), bool))
    seen[19:, 19:] = False
    for i, p in enumerate(parents):
        if p >= 0:
            seen[19 + i, 19:] = seen[19 + p, 19:]
        seen[19 + i, 19 + i] = True
    want = dense_logits(X, model, tokens, list(range(19)) + [19 + d for d in depth], seen)
    got = torch.cat(got).double().cpu()
    assert (got - want).norm() / want.norm() < 5e-3 and (got[19:] - want[19:]).norm() / want[19:].norm() < 5e-3
    # the path 0, 3, 4, 7 of the tree, kept: the caches then hold what a row of these tokens leaves
    path = torch.tensor([[2, 3, 6, -1, -1, -1, -1]], dtype=torch.int32, device="cuda")          # (nodes count from the token behind the one that waits)
    model.keep(19, path, torch.tensor([3], dtype=torch.int32, device="cuda"))
    after = model.logits(tokens[:2], 23)
    row = X.TreeDecoder(bits=16)
    line = tokens[:19] + [tokens[19 + i] for i in (0, 3, 4, 7)]
    for i in range(0, 23, 8):
        row.logits(line[i:min(i + 8, 23)], i)
    same = row.logits(tokens[:2], 23)
    assert (after - same).norm() / same.norm() < 5e-3
