"""The example with drafts that are known: right ones, which are accepted and whose keys and values stay in the cache, and wrong ones among
them, whose places are written again."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("wrong", [None, 0, 3, 6])
def test_accepted_and_refused(monkeypatch, bits, wrong):
    """`wrong`: which of a step's seven drafts is another token.  The answer is that without drafts, in the steps that it takes: a step gives the
    drafts before the wrong one and a token of its own."""
    import drafted_decoding as X
    prompt, count = [int(t) for t in np.random.default_rng(5).integers(0, X.VOCAB, 17)], 41
    plain, steps = X.generate(X.Decoder(bits=bits), prompt, count, drafts=0)
    assert steps == count == len(plain)
    asked = []

    def known(tokens, most):
        at = len(tokens) - len(prompt)
        guess = plain[at:at + most]
        if wrong is not None and wrong < len(guess):
            guess = guess[:wrong] + [(guess[wrong] + 1) % X.VOCAB] + guess[wrong + 1:]
        asked.append((len(guess), wrong is not None and wrong < len(guess)))
        return guess
    monkeypatch.setattr(X, "drafts_for", known)
    drafted, fewer = X.generate(X.Decoder(bits=bits), prompt, count, drafts=7)
    assert drafted == plain
    # each step: all drafts, or those before the wrong one, and one token more
    assert fewer == len(asked) and sum(wrong + 1 if bad else n + 1 for n, bad in asked) == count
    assert fewer < count // 2 if wrong in (None, 3, 6) else fewer >= count - 7
