"""The check of trees of drafted tokens: whole numbers, equal to those of the definition in 64 bits."""
import numpy as np
import pytest
import tree_reference as tree

pytestmark = pytest.mark.gpu


def make(batch, nodes, vocab, seed, sharp=6.0):
    """Trees whose tokens are mostly among the likeliest of their places; some siblings alike, some tokens that are none, some parents that are none."""
    rng = np.random.default_rng(seed)
    a = sharp * rng.normal(size=(batch, nodes + 1, vocab))
    e = np.exp(a - a.max(-1, keepdims=True))
    target = (e / e.sum(-1, keepdims=True)).astype(np.float32)
    parent = np.array([tree.parents(rng, nodes) for _ in range(batch)], np.int32).reshape(batch, nodes)
    drafted = np.zeros((batch, nodes), np.int32)
    for b in range(batch):
        for i in range(nodes):
            order = np.argsort(-target[b, parent[b, i] + 1])
            drafted[b, i] = order[min(int(rng.integers(0, 4)), vocab - 1)]
    wild = rng.random((batch, nodes))
    drafted[wild < 0.04] = rng.choice([-1, -7, vocab, 2 ** 31 - 1])
    parent[(wild > 0.04) & (wild < 0.07)] = rng.choice([-2, nodes, 2 ** 31 - 1, -2 ** 31])
    return target, drafted, parent, rng.random((batch, nodes + 1)).astype(np.float32)


def run(target, drafted, parent, uniform, count=None, pad=0):
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
    out = [torch.full(s, 12345, dtype=torch.int32, device="cuda") for s in (uniform.shape, drafted.shape, uniform.shape[:1])]
    D.verify_tree(put(target), put(drafted), put(parent), put(uniform), *out, put(count))
    return [t.cpu().numpy() for t in out]


def equal(got, want):
    assert all(np.array_equal(g, w) for g, w in zip(got, want)), (got, want)


@pytest.mark.parametrize("batch,nodes,vocab", [(1, 1, 1), (3, 2, 5), (5, 4, 255), (4, 7, 256), (40, 13, 257), (2, 0, 1000), (60, 26, 1024), (6, 63, 4099),
                                               (9, 64, 50), (9, 65, 50), (3, 200, 33), (2, 1024, 40), (3, 20, 32000), (2, 4, 50272), (1, 2, 128256)])
@pytest.mark.parametrize("pad", [0, 3])
def test_against_64_bits(batch, nodes, vocab, pad):
    a = make(batch, nodes, vocab, vocab + nodes)
    want = tree.verify(*a)
    equal(run(*a, pad=pad), want)
    count = np.random.default_rng(7).integers(-1, nodes + 3, batch).astype(np.int32)
    equal(run(*a, count=count, pad=pad), tree.verify(*a, count))


def test_paths_are_long_and_siblings_are_refused():
    """That the cases above hold what they should."""
    _, path, n = tree.verify(*make(60, 26, 1024, 1050))
    assert n.max() >= 3 and (n == 0).any() and any(np.diff(p[:k]).max(initial=0) > 1 for p, k in zip(path, n))


def test_random_numbers_at_their_ends():
    a = make(30, 9, 700, 1)
    for u in (0.0, np.nextafter(np.float32(1), np.float32(0))):
        uniform = np.full_like(a[3], u)
        equal(run(*a[:3], uniform), tree.verify(*a[:3], uniform))


def test_a_tree_without_branches_is_a_row_of_drafts():
    import torch
    from paper_2507_12205_amd import device as D
    target, drafted, _, uniform = make(200, 6, 900, 3)
    parent = np.tile(np.arange(-1, 5, dtype=np.int32), (200, 1))
    tokens, path, accepted = run(target, drafted, parent, uniform)
    other = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((200, 7), (200,))]
    D.verify(*(None if x is None else torch.from_numpy(x).cuda() for x in (target, None, drafted, uniform)), *other)
    assert np.array_equal(tokens, other[0].cpu().numpy()) and np.array_equal(accepted, other[1].cpu().numpy()) and 0 < accepted.mean() < 6
    assert np.array_equal(path, np.where(np.arange(6) < accepted[:, None], np.arange(6), -1))


def test_nothing_left():
    """Certain targets; everything drafted and refused; rows without anything above zero; NaN among the probabilities."""
    target = np.zeros((6, 4, 3), np.float32)
    target[0, :, 1] = 1                                      # certain
    target[1] = 0.25                                         # all three tokens drafted: they take 0.75 in all
    target[2] = 0
    target[3, :, 2], target[3, :, 0] = np.nan, 0.5
    target[4] = -1
    target[5] = [0.5, 0.5, 0.0]
    drafted = np.array([[0, 1, 1], [0, 1, 2], [0, 1, 2], [2, 0, 1], [0, 1, 2], [0, 0, 1]], np.int32)
    parent = np.array([[-1, -1, 1], [-1, -1, -1], [-1, -1, -1], [-1, -1, -1], [-1, 0, 1], [-1, -1, -1]], np.int32)
    for u in (0.0, 0.4, 0.8, 0.999):
        uniform = np.full((6, 4), u, np.float32)
        equal(run(target, drafted, parent, uniform), tree.verify(target, drafted, parent, uniform))


def test_tokens_have_the_target_s_probabilities():
    """65000 draws: each first token's frequency within five standard deviations of its probability, whatever was drafted."""
    rng, n = np.random.default_rng(11), 65000
    p = np.array([0.5, 0.2, 0.15, 0.1, 0.05], np.float32)
    second = np.array([0.05, 0.05, 0.1, 0.2, 0.6], np.float32)
    target = np.ascontiguousarray(np.broadcast_to(np.stack([p, second, p, second, p]), (n, 5, 5)))
    drafted, parent = np.tile(np.array([1, 0, 4, 2], np.int32), (n, 1)), np.tile(np.array([-1, -1, 0, -1], np.int32), (n, 1))
    tokens, path, accepted = run(target, drafted, parent, rng.random((n, 5)).astype(np.float32))
    for v in range(5):
        assert abs((tokens[:, 0] == v).mean() - p[v]) < 5 * (p[v] * (1 - p[v]) / n) ** 0.5
    after = tokens[tokens[:, 0] == 1][:, 1]                  # after node 0, which has a child: whether it is accepted or not
    for v in range(5):
        assert abs((after == v).mean() - second[v]) < 5 * (second[v] * (1 - second[v]) / len(after)) ** 0.5


@pytest.mark.parametrize("batch,nodes,vocab", [(1, 5, 3000), (40, 30, 40000)])
def test_in_a_graph_and_on_another_stream(batch, nodes, vocab):
    import torch
    from paper_2507_12205_amd import device as D
    made = [torch.from_numpy(x).cuda() for x in make(batch, nodes, vocab, 5)]
    out, eager = ([torch.empty(s, dtype=torch.int32, device="cuda") for s in ((batch, nodes + 1), (batch, nodes), (batch,))] for _ in range(2))
    count = torch.full((batch,), nodes, dtype=torch.int32, device="cuda")
    work = torch.empty(D.verify_tree_workspace(batch, nodes, vocab), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    D.verify_tree(*made, *out, count, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.verify_tree(*made, *out, count, work)
    for turn in range(5):
        for have, x in zip(made, make(batch, nodes, vocab, 20 + turn)):
            have.copy_(torch.from_numpy(x))
        count.random_(0, nodes + 1)
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        D.verify_tree(*made, *eager, count, stream=side)
        side.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, eager))
        equal([t.cpu().numpy() for t in out], tree.verify(*(t.cpu().numpy() for t in made), count.cpu().numpy()))


@pytest.mark.parametrize("batch,nodes,vocab", [(1, 7, 50000), (40, 30, 40000), (3, 1024, 9000)])
@pytest.mark.parametrize("outputs", ["count", "parent", "drafted", "all"])
def test_outputs_in_the_inputs_memory(outputs, batch, nodes, vocab):
    """Outputs are written when every walk has ended: they may lie where the tree and its random numbers lie."""
    import torch
    from paper_2507_12205_amd import device as D
    a = make(batch, nodes, vocab, 17)
    lengths = np.random.default_rng(3).integers(nodes // 2, nodes + 1, batch).astype(np.int32)
    want = tree.verify(*a, lengths)
    for turn in range(3):
        target, drafted, parent, uniform, count = (torch.from_numpy(x.copy()).cuda() for x in (*a, lengths))
        tokens, path, accepted = (torch.full(x.shape, 12345, dtype=torch.int32, device="cuda") for x in (uniform, drafted, count))
        if outputs in ("count", "all"):
            accepted = count
        if outputs in ("parent", "all"):
            path = parent
        if outputs == "drafted":
            path = drafted
        if outputs == "all":
            tokens = uniform.view(torch.int32)
        equal([t.cpu().numpy() for t in D.verify_tree(target, drafted, parent, uniform, tokens, path, accepted, count)], want)
