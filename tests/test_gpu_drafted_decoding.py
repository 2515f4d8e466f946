"""The example that runs products with epilogues, cache, attention and check of drafts together: with drafts it says what it says without,
and a step's logits are those of the same decoder in dense 64-bit arithmetic."""
import math
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_drafts_change_nothing(bits):
    import drafted_decoding as X
    prompt = [int(t) for t in np.random.default_rng(3).integers(0, X.VOCAB, 5)] * 3
    plain, steps = X.generate(X.Decoder(bits=bits), prompt, 30, drafts=0)
    assert steps == 30
    # a copy of the answer as part of the prompt makes for good drafts
    drafted, fewer = X.generate(X.Decoder(bits=bits), prompt, 30, drafts=7)
    assert drafted == plain and fewer <= steps
    sampled, _ = X.generate(X.Decoder(bits=bits), prompt, 30, drafts=7, sample=True)
    assert len(sampled) >= 30 and all(0 <= t < X.VOCAB for t in sampled)


def test_logits_against_dense_64_bits():
    """FP16 activations between the operators: every layer rounds some ten times at 2^-11, on values of about 1; a tenth of that in sum."""
    import torch
    import drafted_decoding as X
    model = X.Decoder(bits=16)
    tokens = [int(t) for t in np.random.default_rng(4).integers(0, X.VOCAB, 21)]
    got = torch.cat([model.logits(tokens[i:i + 8], i) for i in range(0, 21, 8)]).double().cpu()
    x = (model.embed[torch.tensor(tokens)] + model.position[:21]).double().cpu()

    def lin(m, v):
        return v @ m.dense.double().t() + m.bias.double().cpu()

    def norm(v):
        return torch.nn.functional.layer_norm(v, (X.HIDDEN,))
    mask = torch.full((21, 21), -math.inf).triu(1).double()
    for layer in model.layers:
        h = norm(x)
        q, k, v = lin(layer["q"], h).view(21, X.HEADS, X.DIM), lin(layer["k"], h).view(21, X.KV_HEADS, X.DIM), lin(layer["v"], h).view(21, X.KV_HEADS, X.DIM)
        k, v = (t.repeat_interleave(X.HEADS // X.KV_HEADS, 1) for t in (k, v))
        s = torch.softmax(torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(X.DIM) + mask, -1)
        x = x + lin(layer["o"], torch.einsum("hij,jhd->ihd", s, v).reshape(21, -1))
        x = x + lin(layer["down"], torch.relu(lin(layer["up"], norm(x))))
    want = lin(model.head, norm(x))
    assert (got - want).norm() / want.norm() < 5e-3
