"""Attention over the paged cache where few and many rows are joined from splits, and NaN and infinities on their way through: every kernel
that a call can take, against 64 bits."""
import numpy as np
import pytest
from test_gpu_attention import check, make, run

pytestmark = pytest.mark.gpu

# how the result comes about: new tokens and keys of each sequence, heads, heads of the cache, dim, page
WAYS = {
    "16 rows, whole": ([2, 1], [100, 31], 4, 2, 64, 16),
    "128 rows, whole": ([150], [200], 2, 2, 64, 16),
    "16 rows, few joined": ([2], [1000], 4, 2, 64, 16),
    "128 rows, few joined": ([150], [900], 2, 2, 96, 32),
    "16 rows, many joined, 64": ([1] * 36, [600 - 9 * i for i in range(36)], 64, 8, 64, 16),
    "16 rows, many joined, 128": ([1] * 40, [300 + 11 * i for i in range(40)], 64, 8, 128, 32),
    "16 rows, many joined, 80": ([2] * 20, [513 - 7 * i for i in range(20)], 64, 8, 80, 16),
    "128 rows, many joined, 48": ([300, 280], [700, 281], 4, 2, 48, 64),
    "128 rows, many joined, 128": ([300, 280], [300, 999], 4, 4, 128, 16),
    "128 rows, many joined, 256": ([300, 280], [700, 300], 4, 2, 256, 16),
    "128 rows, many joined, 240": ([600], [900], 4, 1, 240, 16),
}


def way(name, bits, seed, torch):
    """The call, after a look at whether it goes that way."""
    from paper_2507_12205_amd import binding as B, device as D
    new, total, heads, kv_heads, dim, page = case = WAYS[name]
    made = make(torch, D, *case, bits, seed=seed)
    a = B.AttentionDesc(D._ATTENTION, heads, sum(new), len(new), made[4].shape[1], max(new))
    assert (B.ecspmv_attention_workspace(made[0].desc, a) > 0) == ("whole" not in name)
    assert (sum(new) * heads >= 2048) == ("many" in name) and (max(new) * heads // kv_heads > 64) == ("128 rows" in name)
    return made


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("name", WAYS)
def test_against_64_bits(name, bits):
    import torch
    from paper_2507_12205_amd import device as D
    made = way(name, bits, 21, torch)
    check(run(torch, D, *made), *made)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("name", WAYS)
def test_nan_in_a_query(name, bits):
    """A query with a NaN has NaN for a result, and no other row has."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, total, table = way(name, bits, 22, torch)
    clean = run(torch, D, cache, q, start, total, table)
    rows = [(0, 1), (q.shape[0] - 1, 0), (q.shape[0] // 2, q.shape[1] - 1)]
    for t, h in rows:
        q[t, h, 3] = float("nan")
    got = run(torch, D, cache, q, start, total, table)
    for t, h in rows:
        assert np.isnan(got[t, h]).all()
        got[t, h] = clean[t, h]
    assert np.array_equal(got, clean)


@pytest.mark.parametrize("name", [n for n in WAYS if "joined" in n])
def test_nan_in_all_keys_of_a_split(name):
    """256 keys of NaN, that is of one split at most two: the rows that see them have NaN for a result."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, total, table = way(name, 16, 23, torch)
    clean = run(torch, D, cache, q, start, total, table)
    for i in range(256):
        cache.k[int(table[0, i // cache.page_size]), 0, i % cache.page_size] = float("nan")
    got = run(torch, D, cache, q, start, total, table)
    group, end = q.shape[1] // cache.heads, int(start[1])
    assert np.isnan(got[:end, :group]).all()
    got[:end, :group] = clean[:end, :group]
    assert np.array_equal(got, clean)


@pytest.mark.parametrize("scale", [None, 4.0])
@pytest.mark.parametrize("name", WAYS)
def test_values_that_are_not_finite(name, scale):
    """Softmax's weights are above zero, however small they come out (the scale of 4: most of them below what FP16 or FP32 hold): an infinity in a
    value that a row sees is its result, two of different sign or a NaN make NaN; other rows, heads and columns keep their bits."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, total, table = way(name, 16, 24, torch)
    clean = run(torch, D, cache, q, start, total, table, scale=scale)
    inf = float("inf")
    odd = [(0, 5, inf), (2, 5, inf), (7, 6, -inf), (9, 8, inf), (11, 8, -inf), (12, 9, float("nan")), (30, 11, -inf), (int(total[0]) - 1, 12, inf)]
    for key, d, x in odd:
        cache.v[int(table[0, key // cache.page_size]), 0, key % cache.page_size, d] = x
    want, group = clean.copy(), q.shape[1] // cache.heads
    for t in range(int(start[1])):
        seen = int(total[0] - start[1]) + t + 1
        for d in {d for _, d, _ in odd}:
            met = [x for key, e, x in odd if e == d and key < seen]
            if met:
                want[t, :group, d] = sum(met)
    got = run(torch, D, cache, q, start, total, table, scale=scale)
    assert np.array_equal(got, want, equal_nan=True)
