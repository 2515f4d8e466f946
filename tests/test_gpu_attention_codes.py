"""Attention over a cache in 8 and 4 bits: values whose steps lie far apart, and queries whose values do not cancel.

The bound, with p the softmax's weights, v a key's values as the cache holds them and top_j the largest |v| of key j: the result is FP16 (2^-11
of it), weights times steps are FP16 (2^-11 of every p_j |v_j|; below the normal range 2^-25 of the largest p_j times step, 127 steps or 8
of 15 making up top_j), FP32 elsewhere (2^-14 of the terms covers sums and exponentials).  4 bits: a value is split in the middle of its row's
reach and a whole number of steps, both up to 2.1 top_j.  Scores in FP32: off by 2^-22 of scale times sum |q| times the key's largest value (a sum of
dim products, with 4 bits of its two parts), which p doubles."""
import numpy as np
import pytest
import serve_reference as ref
from test_gpu_attention import make, run, values

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def seed():
    import torch
    torch.manual_seed(1)


def bound(cache, q, start, total, table, scale, weights=2 ** -11):
    """(result in 64 bits, bound of the error); weights: how far those of 16 bits are off"""
    k, v = values(cache)
    q = q.cpu().numpy().astype(np.float64)
    want, slack = np.zeros(q.shape), np.zeros(q.shape)
    group, parts = q.shape[1] // k.shape[1], 2.1 if cache.bits == 4 else 1.0
    for b, n in enumerate(total):
        kk, vv = ref.gather(k, table[b], n), ref.gather(v, table[b], n)
        new = start[b + 1] - start[b]
        for t in range(new):
            seen = n - new + t + 1
            for h in range(q.shape[1]):
                x, kr, vr = q[start[b] + t, h], kk[h // group, :seen], vv[h // group, :seen]
                a = scale * (kr @ x)
                p = np.exp(a - a.max())
                p /= p.sum()
                top = np.abs(vr).max(1)
                size = p @ np.abs(vr) if cache.bits == 8 else np.full(x.shape, parts * (p @ top))
                score = 2 ** -22 * scale * np.abs(x).sum() * parts * np.abs(kr).max()
                want[start[b] + t, h] = o = p @ vr
                slack[start[b] + t, h] = 2 ** -11 * np.abs(o) + (weights + 2 ** -14 + 2 * score) * size + seen * 2 ** -24 * parts * (p * top).max() + 2 ** -25
    return want, slack


def encode(x, bits, torch):
    """(codes, steps) of (..., dim) values, as kv_write makes them."""
    from paper_2507_12205_amd import device as D
    flat = x.reshape(-1, 1, x.shape[-1])
    cache = D.kv_cache(-(-flat.shape[0] // 16), 1, 16, x.shape[-1], bits)
    D.kv_write(cache, flat, flat, torch.arange(flat.shape[0], device="cuda"))
    return [t.transpose(1, 2).reshape(-1, *t.shape[3:])[:flat.shape[0]] for t in (cache.v, cache.v_step)]


def put_value(cache, table, key, head, x, torch):
    page, off = int(table[0, key // cache.page_size]), key % cache.page_size
    code, step = encode(x[None, None], cache.bits, torch)
    cache.v[page, head, off], cache.v_step[page, head, off] = code[0], step[0]


SHAPES = [(6, 70), (40, 200), (200, 330), (6, 3000), (1, 500), (130, 900)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,total", SHAPES[:4])
@pytest.mark.parametrize("odd", [float("inf"), -60000.0])
def test_values_that_later_tokens_only_see(new, total, odd, bits):
    """A large value of a later token changes no bit of the tokens that do not see it."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = make(torch, D, [new], [total], 4, 2, 128, 16, bits, seed=4)
    clean = run(torch, D, cache, q, start, lens, table)
    at = total - new // 2
    first = at - (total - new)
    x = torch.randn(128, device="cuda").half()
    x[5] = odd
    put_value(cache, table, at, 1, x, torch)
    got = run(torch, D, cache, q, start, lens, table)
    assert np.array_equal(got[:first], clean[:first]) and np.array_equal(got[:, :2], clean[:, :2])
    want, slack = bound(cache, q, start, lens, table, 128 ** -0.5)
    assert (np.abs(got - want) <= slack).all()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,total", SHAPES)
def test_a_large_value_without_weight(new, total, bits):
    """A key that all see, with values of up to 60000 and a score some 60 below the rest."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = make(torch, D, [new], [total], 4, 2, 128, 16, bits, seed=5)
    q += 4                                                   # (so that a key of equal values has a score of its own)
    for at in (3, 17):
        put_value(cache, table, at, 1, (30000 * torch.rand(128, device="cuda") + 30000).half() * torch.randn(128, device="cuda").sign().half(), torch)
        page, off = int(table[0, at // 16]), at % 16
        code, step = encode(torch.linspace(-1.6, -1.4, 128, device="cuda").half()[None, None], bits, torch)
        cache.k[page, 1, off], cache.k_step[page, 1, off] = code[0], step[0]
    got = run(torch, D, cache, q, start, lens, table)
    want, slack = bound(cache, q, start, lens, table, 128 ** -0.5)
    worst = np.max(np.abs(got - want) / slack)
    assert worst <= 1, worst


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,total", SHAPES)
def test_values_of_all_sizes(new, total, bits):
    """Rows of V from 2^-20 to 2^12, rows of zeros and of one value among them, and none but zeros in the first keys."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = make(torch, D, [new], [total], 4, 2, 128, 16, bits, seed=6)
    rng = np.random.default_rng(7)
    for at in range(min(total, 160)):
        x = torch.randn(128, device="cuda") * float(2.0 ** rng.integers(-20, 13))
        if at < 66 or at % 7 == 0:
            x = torch.zeros(128, device="cuda")
        elif at % 7 == 1:
            x = torch.full((128,), float(rng.normal()), device="cuda")
        for head in range(2):
            put_value(cache, table, at, head, x.half(), torch)
    got = run(torch, D, cache, q, start, lens, table)
    want, slack = bound(cache, q, start, lens, table, 128 ** -0.5)
    worst = np.max(np.abs(got - want) / slack)
    assert worst <= 1, worst


@pytest.mark.parametrize("bits", [8, 4])
def test_both_parts_of_a_weight(bits):
    """50000 rows of three keys: the two FP16 parts of every weight times step (2^-21 of it together) belong to one another, also where the
    weight lies between two FP16 values."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = make(torch, D, [1] * 800, [3] * 800, 64, 8, 64, 16, bits, seed=9)
    got = run(torch, D, cache, q, start, lens, table)
    want, slack = bound(cache, q, start, lens, table, 0.125, 2 ** -21)
    worst = np.max(np.abs(got - want) / slack)
    assert worst <= 1, worst


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("queries", ["of mean 6", "of a few large channels"])
@pytest.mark.parametrize("new,total,heads,dim", [(1, 2, 64, 128), (2, 3, 32, 64), (1, 12, 64, 128), (2, 4, 16, 256), (3, 5, 8, 96), (150, 150, 2, 128)])
def test_queries_that_do_not_cancel(new, total, heads, dim, queries, bits):
    """Scores are as exact as sums of FP32 over the codes: nothing much larger than those is added up and taken off again.  (The weights of the
    kernel for few rows are FP16 in two parts: 2^-21.)"""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = make(torch, D, [new] * 40, [total] * 40, heads, heads // 2, dim, 16, bits, seed=8)
    if queries == "of mean 6":
        q = (0.5 * q + 6).half()
    else:
        q = (q * torch.where(torch.rand(dim, device="cuda") < 0.04, 20.0, 1.0)).half()
    got = run(torch, D, cache, q, start, lens, table)
    want, slack = bound(cache, q, start, lens, table, dim ** -0.5, 2 ** -11 if new > 100 else 2 ** -21)
    worst = np.max(np.abs(got - want) / slack)
    assert worst <= 1, worst
