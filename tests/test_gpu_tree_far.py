"""Decoding with trees where offsets pass 32 bits: the last pages of a cache of 4.7 GB each for keys and values, rows of probabilities 8.6 GB apart."""
import numpy as np
import pytest
import tree_reference as tree
from test_gpu_kv_cache import values
from test_gpu_verify_tree import make

pytestmark = pytest.mark.gpu


def test_the_last_pages_of_a_large_cache():
    """Appended, attended and kept there as in a small cache."""
    import torch
    from paper_2507_12205_amd import device as D
    pages, heads, page, dim = 9100, 8, 256, 128
    large, small = (D.KvCache(*(torch.empty((n, heads, page, dim), dtype=torch.float16, device="cuda") for _ in range(2))) for n in (pages, 4))
    assert large.k.nbytes > 1 << 32
    k, v, q = values((300, heads, dim), 1, torch), values((300, heads, dim), 2, torch), values((300, 2 * heads, dim), 3, torch)
    at, position, freq = torch.arange(300, device="cuda"), torch.arange(300, dtype=torch.int32, device="cuda"), D.rotary_frequency(64)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")        # noqa: E731
    parents = tree.parents(np.random.default_rng(3), 40)
    path = [i for i in range(40) if tree.tree_seen(parents)[39][i]]
    assert len(path) > 2
    out = []
    for cache, first in ((large, pages - 4), (small, 0)):
        table = i32([[first + 3, first + 1]])
        slots = table[0].long()[at // page] * page + at % page
        turned = D.kv_append(cache, k, v, slots, position, freq, q, torch.empty_like(q))
        news = turned[260:]
        o = D.attention_tree(cache, news, torch.empty_like(news), i32([0, 40]), i32([300]), table, D.tree_seen([parents]), 40)
        D.kv_keep(D.KvCaches([cache]), i32([260]), i32([path]), i32([len(path)]), table)
        out.append([turned, o, cache.k[first + 1].clone(), cache.v[first + 1].clone(), cache.k[first + 3].clone(), cache.v[first + 3].clone()])
    # (pages that were not written hold anything: their first 300 places are compared)
    for i, (x, y) in enumerate(zip(*out)):
        n = x.shape[1] if i < 2 or i > 3 else 300 - page
        assert torch.equal(x[:, :n], y[:, :n])


def test_probabilities_that_lie_far_apart():
    import torch
    from paper_2507_12205_amd import device as D
    target, drafted, parent, uniform = make(2, 9, 700, 4)
    apart = (1 << 31) + 5
    memory = torch.empty(apart + 10 * 700, dtype=torch.float32, device="cuda")
    far = memory.as_strided((2, 10, 700), (apart, 700, 1))
    far.copy_(torch.from_numpy(target))
    out = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((2, 10), (2, 9), (2,))]
    D.verify_tree(far, *(torch.from_numpy(x).cuda() for x in (drafted, parent, uniform)), *out)
    for got, want in zip(out, tree.verify(target, drafted, parent, uniform)):
        assert np.array_equal(got.cpu().numpy(), want)
