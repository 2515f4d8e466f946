"""The check of drafted tokens: whole numbers, equal to those of the definition in 64 bits."""
import numpy as np
import pytest
import serve_reference as ref

pytestmark = pytest.mark.gpu


def make(batch, drafts, vocab, seed, sharp=2.0):
    rng = np.random.default_rng(seed)

    def soft(x):
        e = np.exp(x - x.max(-1, keepdims=True))
        return (e / e.sum(-1, keepdims=True)).astype(np.float32)
    a = sharp * rng.normal(size=(batch, drafts + 1, vocab))
    target, draft = soft(a), soft(a[:, :drafts] + 0.5 * rng.normal(size=(batch, drafts, vocab)))
    drafted = np.array([[rng.choice(vocab, p=draft[b, i].astype(np.float64) / draft[b, i].sum(dtype=np.float64)) for i in range(drafts)]
                        for b in range(batch)], np.int32).reshape(batch, drafts)
    return target, draft, drafted, rng.random((batch, drafts + 1)).astype(np.float32)


def run(target, draft, drafted, uniform, count=None, pad=0):
    import torch
    from paper_2507_12205_amd import device as D

    def put(x):
        if x is None:
            return None
        if pad and x.ndim == 3:                              # rows and sequences apart, and off 16 bytes
            wide = torch.full((x.shape[0], x.shape[1] + 1, x.shape[2] + pad), 9.0, device="cuda")
            wide[:, :x.shape[1], 1:x.shape[2] + 1] = torch.from_numpy(x).cuda()
            return wide[:, :x.shape[1], 1:x.shape[2] + 1]
        return torch.from_numpy(x).cuda()
    tokens = torch.full(uniform.shape, 12345, dtype=torch.int32, device="cuda")
    accepted = torch.full((len(uniform),), 12345, dtype=torch.int32, device="cuda")
    D.verify(put(target), put(draft), put(drafted), put(uniform), tokens, accepted, put(count))
    return tokens.cpu().numpy(), accepted.cpu().numpy()


def equal(got, want):
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[0], want[0]), (got, want)


@pytest.mark.parametrize("batch,drafts,vocab", [(1, 1, 1), (3, 2, 5), (5, 4, 255), (4, 7, 256), (4, 3, 257), (2, 0, 1000), (6, 5, 4099), (3, 7, 32000),
                                                (2, 2, 50272), (1, 1, 128256), (9, 70, 33)])
@pytest.mark.parametrize("pad", [0, 3])
def test_against_64_bits(batch, drafts, vocab, pad):
    a = make(batch, drafts, vocab, vocab + drafts)
    equal(run(*a, pad=pad), ref.verify(*a))
    target, _, drafted, uniform = a
    equal(run(target, None, drafted, uniform, pad=pad), ref.verify(target, None, drafted, uniform))
    count = np.random.default_rng(7).integers(0, drafts + 1, batch).astype(np.int32)
    equal(run(*a, count=count, pad=pad), ref.verify(*a, count))


def test_random_numbers_at_their_ends():
    a = make(4, 3, 700, 1)
    for u in (0.0, np.nextafter(np.float32(1), np.float32(0))):
        uniform = np.full_like(a[3], u)
        equal(run(*a[:3], uniform), ref.verify(*a[:3], uniform))


def test_nothing_left_and_nothing_at_all():
    """Where the draft says the same as the target and is refused all the same (a drafted token that is none): from the target; a row of
    zeros has no next token; NaN counts as 0."""
    target, draft, drafted, uniform = make(4, 2, 300, 2)
    draft[:, 0] = target[:, 0]
    drafted[0, 0], drafted[1, 0], drafted[2, 0], drafted[3, 0] = -1, 300, 2 ** 31 - 1, -2 ** 31
    equal(run(target, draft, drafted, uniform), ref.verify(target, draft, drafted, uniform))
    equal(run(target, None, drafted, uniform), ref.verify(target, None, drafted, uniform))
    target[1, 0] = 0
    target[2, 0, 5] = np.nan
    got = run(target, draft, drafted, uniform)
    equal(got, ref.verify(target, draft, drafted, uniform))
    assert got[0][1, 0] == -1


def test_probabilities_all_on_a_few_tokens():
    """one token, and the first and the last of a tile of 256 and of the vocabulary"""
    vocab = 1025
    for places in ([0], [1024], [255, 256], [0, 1024], [511, 512, 1023]):
        target = np.zeros((8, 2, vocab), np.float32)
        target[:, :, places] = 1 / len(places)
        draft = np.full((8, 1, vocab), 1 / vocab, np.float32)
        drafted = np.full((8, 1), 77, np.int32)
        uniform = np.random.default_rng(3).random((8, 2)).astype(np.float32)
        equal(run(target, draft, drafted, uniform), ref.verify(target, draft, drafted, uniform))


def test_shares_follow_the_target():
    """Accepted or drawn after a refusal, the first token is the target's: 40000 trials over 6 tokens, within five standard deviations."""
    rng = np.random.default_rng(5)
    n, p, q = 40000, np.array([0.4, 0.25, 0.2, 0.1, 0.05, 0.0]), np.array([0.1, 0.1, 0.3, 0.2, 0.1, 0.2])
    target = np.broadcast_to(p.astype(np.float32), (n, 2, 6)).copy()
    draft = np.broadcast_to(q.astype(np.float32), (n, 1, 6)).copy()
    drafted = rng.choice(6, size=(n, 1), p=q).astype(np.int32)
    tokens, _ = run(target, draft, drafted, rng.random((n, 2)).astype(np.float32))
    share = np.bincount(tokens[:, 0], minlength=6) / n
    assert (np.abs(share - p) <= 5 * np.sqrt(p * (1 - p) / n) + 1e-9).all()
