"""Rows of accepted nodes moved to where they follow one another: bits are copied as they are, and nothing else changes."""
import numpy as np
import pytest
import tree_reference as tree

pytestmark = pytest.mark.gpu


def caches(torch, D, layers, pages, heads, page, dim, bits, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    made = [D.kv_cache(pages, heads, page, dim, bits) for _ in range(layers)]
    for c in made:
        for t in tensors(c):
            if t.dtype.is_floating_point:
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
            else:
                t.random_(-128 if t.dtype is torch.int8 else 0, 127 if t.dtype is torch.int8 else 255, generator=g)
    return made


def tensors(c):
    return [t for t in (c.k, c.v, c.k_step, c.v_step) if t is not None]


def check(torch, D, made, first, path, accepted, table, stream=None):
    want = [[t.cpu().numpy().copy() for t in tensors(c)] for c in made]
    for w in want:
        tree.keep(w, first, path, accepted, table, made[0].page_size)
    D.kv_keep(D.KvCaches(made), *(torch.from_numpy(x).cuda() for x in (first, path, accepted, table)), stream=stream)
    torch.cuda.synchronize()
    for c, w in zip(made, want):
        for t, x in zip(tensors(c), w):
            assert np.array_equal(t.cpu().numpy().view(np.uint8), x.view(np.uint8))


def growing(rng, nodes, n):
    return np.sort(rng.choice(nodes, n, replace=False))


# layers, batch, nodes, heads, dim, page
SHAPES = [(1, 1, 1, 1, 16, 16), (3, 2, 8, 2, 64, 16), (2, 5, 63, 8, 128, 64), (5, 3, 26, 5, 80, 32), (2, 1, 40, 3, 256, 16), (1, 2, 700, 1, 48, 16)]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows_move(shape, bits):
    import torch
    from paper_2507_12205_amd import device as D
    layers, batch, nodes, heads, dim, page = shape
    rng = np.random.default_rng(nodes)
    past = rng.integers(0, 3 * page, batch)
    need = [-(-(int(p) + nodes) // page) for p in past]
    pages = sum(need) + 2
    order, table, at = rng.permutation(pages), np.full((batch, max(need) + 1), -7, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    made = caches(torch, D, layers, pages, heads, page, dim, bits, nodes)
    for turn in range(3):                                    # some, all in place, none
        accepted = np.array([int(rng.integers(0, nodes + 1)) for _ in range(batch)], np.int32) if turn < 2 else np.zeros(batch, np.int32)
        path = np.full((batch, nodes), -1, np.int32)
        for b, n in enumerate(accepted):
            path[b, :n] = growing(rng, nodes, n) if turn == 0 else np.arange(n)
        check(torch, D, made, past.astype(np.int32), path, accepted, table)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_what_is_out_of_place_stays(bits):
    """Places beyond the table, pages that are none, nodes before their place, counts below 0 and beyond the nodes."""
    import torch
    from paper_2507_12205_amd import device as D
    made = caches(torch, D, 2, 6, 2, 16, 32, bits, 5)
    table = np.array([[0, 1, 2], [3, -1, 4], [5, 2 ** 31 - 1, 6]], np.int32)
    first = np.array([30, 10, 0], np.int32)
    path = np.array([[1, 3, 17, 18, 40, 2 ** 31 - 1], [2, 3, 5, 9, 30, 36], [4, 1, -1, 5, 33, 47]], np.int32)
    check(torch, D, made, first, path, np.array([6, 99, 6], np.int32), table)
    check(torch, D, made, np.array([-3, 47, 2 ** 31 - 1], np.int32), path, np.array([6, 6, 6], np.int32), table)
    check(torch, D, made, first, path, np.array([-1, 0, -2 ** 31], np.int32), table)


def test_many_layers():
    """More caches than one launch takes."""
    import torch
    from paper_2507_12205_amd import device as D
    made = caches(torch, D, 131, 3, 1, 16, 16, 4, 7)
    check(torch, D, made, np.array([3], np.int32), np.array([[2, 4, 9, 20]], np.int32), np.array([4], np.int32), np.array([[2, 0]], np.int32))


def test_strides_streams_and_a_graph():
    import torch
    from paper_2507_12205_amd import device as D
    made = caches(torch, D, 3, 8, 2, 16, 64, 8, 9)
    rng, side = np.random.default_rng(1), torch.cuda.Stream()
    wide_path, wide_table = torch.full((2, 11), -9, dtype=torch.int32, device="cuda"), torch.full((2, 7), -9, dtype=torch.int32, device="cuda")
    table = np.array([[0, 5, 2], [3, 1, 7]], np.int32)
    wide_table[:, :3] = torch.from_numpy(table).cuda()
    first, accepted = (torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2))
    handle = D.KvCaches(made)
    D.kv_keep(handle, first, wide_path[:, :9], accepted, wide_table[:, :3])                  # (nothing is accepted)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.kv_keep(handle, first, wide_path[:, :9], accepted, wide_table[:, :3])
    for turn in range(6):
        n = rng.integers(0, 6, 2)
        f = rng.integers(0, 30, 2).astype(np.int32)
        path = np.stack([np.concatenate([growing(rng, 9, k), np.full(9 - k, -1)]) for k in n]).astype(np.int32)
        first.copy_(torch.from_numpy(f)), accepted.copy_(torch.from_numpy(n.astype(np.int32))), wide_path[:, :9].copy_(torch.from_numpy(path))
        want = [[t.cpu().numpy().copy() for t in tensors(c)] for c in made]
        for w in want:
            tree.keep(w, f, path, n, table, 16)
        torch.cuda.synchronize()
        if turn % 2:
            D.kv_keep(handle, first, wide_path[:, :9], accepted, wide_table[:, :3], stream=side)
        else:
            graph.replay()
        torch.cuda.synchronize()
        for c, w in zip(made, want):
            for t, x in zip(tensors(c), w):
                assert np.array_equal(t.cpu().numpy(), x)
