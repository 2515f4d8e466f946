"""Attention of the nodes of trees over the paged cache against 64 bits: trees and other masks of what new tokens see of one another, what lies in
places that a token does not see, rows that see nothing.  The bound is that of test_gpu_attention."""
import numpy as np
import pytest
import tree_reference as tree
import serve_reference as ref
from test_gpu_attention import make, place, values

pytestmark = pytest.mark.gpu


def trees(rng, new):
    return [tree.tree_seen(tree.parents(rng, n)) for n in new]


def words_of(seen, extra=0, rng=None):
    """The rows of all sequences, `extra` words beyond the widest (and bits of new tokens that there are none of) of any content."""
    words = max([1] + [-(-s.shape[0] // 32) for s in seen]) + extra
    out = np.zeros((sum(s.shape[0] for s in seen), words), np.uint32)
    at = 0
    for s in seen:
        n = s.shape[0]
        if rng is not None:
            wild = rng.random((n, 32 * words)) < 0.5
            wild[:, :n] = s
            s = wild
        out[at:at + n, :max(1, -(-s.shape[1] // 32))] = tree.pack(s).view(np.uint32)[:n] if n else 0
        at += n
    return out.view(np.int32)


def run(torch, D, cache, q, start, total, table, words, layout="tokens", scale=None, workspace="own", max_new=None):
    out = place(torch.full_like(q, float("nan")), layout, torch)
    args = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (start, total, table, words)]
    most = int(np.diff(start).max()) if max_new is None else max_new
    ws = D.attention_workspace(cache, q, len(total), most, table.shape[1] * cache.page_size) if workspace == "own" else workspace
    if ws is not None and ws.numel():
        ws.fill_(255)
    D.attention_tree(cache, place(q, layout, torch), out, *args, most, scale, ws)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64)


def check(got, made, seen, scale=None):
    cache, q, start, total, table = made
    k, v = values(cache)
    want, size = tree.attention(q.cpu().numpy().astype(np.float64), k, v, start, total, table, seen, cache.head_dim ** -0.5 if scale is None else scale)
    assert np.isfinite(got).all()
    top = max((np.abs(ref.gather(v, table[b], n)).max() for b, n in enumerate(total) if n), default=0.0)
    bound = 2 ** -11 * np.abs(want) + (2 ** -11 + 2 ** -14) * (size + (top if cache.bits == 4 else 0.0)) + max(total) * 2 ** -24 * top + 2 ** -25
    worst = np.max(np.abs(got - want) / bound) if got.size else 0.0
    assert worst <= 1.0, worst


CASES = [
    # new tokens and keys of each sequence, heads, heads of the cache, dim, page
    ([1], [1], 1, 1, 16, 16), ([2], [2], 4, 2, 64, 16), ([8], [8], 4, 4, 64, 16), ([16], [300], 12, 12, 64, 16), ([33], [2049], 8, 1, 128, 64),
    ([8], [1000], 4, 4, 128, 32), ([3, 1, 7, 2], [3, 17, 260, 513], 8, 2, 128, 16), ([17, 40], [17, 333], 6, 2, 80, 32),
    ([130], [130], 2, 1, 96, 16), ([65, 1, 33], [700, 1, 33], 4, 4, 64, 128), ([5], [4100], 2, 2, 256, 256), ([200], [456], 3, 3, 128, 64),
    ([31, 32], [100, 63], 16, 1, 240, 16), ([70], [71], 5, 5, 48, 1024), ([64], [1025], 2, 2, 128, 16), ([300], [999], 4, 1, 64, 32),
    ([40], [500], 4, 4, 160, 16), ([20, 50], [300, 800], 2, 2, 192, 16), ([100], [400], 2, 1, 224, 32), ([60], [1200], 8, 8, 32, 16),
    ([9, 30, 2, 0, 1], [3000, 700, 5, 40, 2100], 4, 4, 128, 16), ([3, 5, 1] * 30, [900, 5, 300] * 30, 4, 2, 64, 16),
    ([50, 1] * 32, [60, 600] * 32, 2, 2, 64, 16), ([130, 260], [2000, 900], 2, 2, 128, 64),
    ([40, 3], [300, 2000], 2, 2, 256, 16), ([64], [5000], 3, 3, 256, 64),
]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("case", CASES)
def test_trees(case, bits):
    import torch
    from paper_2507_12205_amd import device as D
    rng = np.random.default_rng(CASES.index(case))
    made = make(torch, D, *case, bits, seed=CASES.index(case), stale=float("nan"))
    seen = trees(rng, case[0])
    check(run(torch, D, *made, words_of(seen)), made, seen)
    check(run(torch, D, *made, words_of(seen, 2, rng)), made, seen)          # words and bits beyond the new tokens: anything


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new,total", [([7, 40], [300, 45]), ([150, 3], [1150, 3])])
def test_any_mask(new, total, bits):
    """Later tokens too, not itself, everything, nothing."""
    import torch
    from paper_2507_12205_amd import device as D
    rng = np.random.default_rng(new[0])
    made = make(torch, D, new, total, 8, 4, 128, 32, bits, seed=3, stale=float("nan"))
    for share in (0.0, 0.1, 0.7, 1.0):
        seen = [rng.random((n, n)) < share for n in new]
        got = run(torch, D, *made, words_of(seen))
        check(got, made, seen)
        if share == 0.0 and total[1] == new[1]:
            assert not got[new[0]:].any()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("layout", ["columns", "odd", "heads"])
@pytest.mark.parametrize("new,total", [([8], [300]), ([150, 3], [150, 90])])
def test_layouts(layout, bits, new, total):
    import torch
    from paper_2507_12205_amd import device as D
    made = make(torch, D, new, total, 8, 4, 128, 32, bits, seed=3, stale=float("inf"))
    words = words_of(trees(np.random.default_rng(1), new))
    assert np.array_equal(run(torch, D, *made, words, layout=layout), run(torch, D, *made, words))


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_rows_that_see_nothing(bits):
    """More new tokens than keys (the first ones have none); sequences without tokens, and without keys; rows without a bit and without a past."""
    import torch
    from paper_2507_12205_amd import device as D
    rng, new = np.random.default_rng(5), [5, 0, 2, 40, 20, 150]
    made = make(torch, D, new, [3, 20, 0, 30, 20, 150], 4, 2, 64, 16, bits, seed=9, stale=float("nan"))
    seen = trees(rng, new)
    seen[4][3], seen[5][149] = False, False
    got = run(torch, D, *made, words_of(seen))
    assert not got[5:7].any() and not got[50].any() and not got[-1].any()
    check(got, made, seen)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new,total", [(6, 70), (40, 200), (200, 330), (7, 3000)])
def test_a_row_of_the_whole_past_only(new, total, bits):
    """No new token seen: what attention gives of one new token before them."""
    import torch
    from paper_2507_12205_amd import device as D
    made = make(torch, D, [new], [total], 4, 2, 128, 16, bits, seed=4, stale=float("nan"))
    seen = [np.zeros((new, new), bool)]
    check(run(torch, D, *made, words_of(seen)), made, seen)


@pytest.mark.parametrize("new,total", [(6, 70), (40, 200), (200, 330), (6, 3000)])
@pytest.mark.parametrize("odd", [float("nan"), float("inf")])
def test_values_that_other_branches_see(new, total, odd):
    """An infinity or NaN in a node's key or value stays with the nodes that see it."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = made = make(torch, D, [new], [total], 4, 2, 128, 16, 16, seed=4)
    seen = trees(np.random.default_rng(new), [new])
    words = words_of(seen)
    clean = run(torch, D, *made, words)
    node = new // 2
    at = total - new + node
    page, off = int(table[0, at // 16]), at % 16
    sees = seen[0][:, node]
    assert sees.any() and not sees.all()
    for tensor in (cache.v, cache.k):
        keep = tensor[page, 1, off, 5].clone()
        tensor[page, 1, off, 5] = odd
        got = run(torch, D, *made, words)
        assert np.array_equal(got[~sees], clean[~sees]) and np.array_equal(got[:, :2], clean[:, :2])
        if tensor is cache.v:
            rest = [d for d in range(128) if d != 5]
            assert np.allclose(got[:, :, rest], clean[:, :, rest], rtol=2 ** -9, atol=2 ** -12)
            assert not np.isfinite(got[sees][:, 2:, 5]).any()
        else:
            assert odd == float("inf") or not np.isfinite(got[sees][:, 2:]).any()
        tensor[page, 1, off, 5] = keep


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,total", [(6, 70), (40, 200), (200, 330)])
def test_nodes_that_were_left_out(new, total, bits):
    """A node that nobody sees may have a row that was never written: steps of NaN, any codes."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = made = make(torch, D, [new], [total], 4, 2, 128, 16, bits, seed=4)
    seen = trees(np.random.default_rng(new), [new])
    node = new // 2
    seen[0][:, node] = False
    words = words_of(seen)
    clean = run(torch, D, *made, words)
    check(clean, made, seen)
    at = total - new + node
    page, off = int(table[0, at // 16]), at % 16
    for odd in (float("nan"), float("inf"), -60000.0):
        for code, step in ((cache.k, cache.k_step), (cache.v, cache.v_step)):
            code[page, :, off], step[page, :, off] = 77, odd
        assert np.array_equal(run(torch, D, *made, words), clean)


@pytest.mark.parametrize("new,total", [(6, 90), (17, 90), (30, 400), (30, 3000), (60, 400)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_infinities_that_rows_see(new, total, dim):
    """A value's infinity is the result of the rows that see it, whatever its weight, zero in FP16 or with a second part below zero; the other values are a mean
    of finite ones.  A key before the tree and a node, one that counts and one that does not."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = made = make(torch, D, [new], [total], 4, 2, dim, 16, 16, seed=4)
    seen = trees(np.random.default_rng(new), [new])
    words = words_of(seen)
    clean = run(torch, D, *made, words)
    for at in (3, total - new - 1, total - new + new // 2):
        page, off = int(table[0, at // 16]), at % 16
        sees = seen[0][:, at - (total - new)] if at >= total - new else np.ones(new, bool)
        assert sees.any()
        for odd in (float("inf"), float("-inf"), float("nan")):
            keep = cache.v[page, 1, off, 7].clone()
            cache.v[page, 1, off, 7] = odd
            got = run(torch, D, *made, words)
            cache.v[page, 1, off, 7] = keep
            assert np.array_equal(got[~sees], clean[~sees]) and np.array_equal(got[:, :2], clean[:, :2])
            assert np.array_equal(got[sees][:, 2:, 7], np.full((sees.sum(), 2), odd), equal_nan=True)
            rest = [d for d in range(dim) if d != 7]
            assert np.array_equal(got[..., rest], clean[..., rest])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,total", [(6, 70), (30, 200), (40, 200), (200, 330), (7, 3000), (100, 3000)])
def test_steps_that_are_none(new, total, bits):
    """A step or lowest value that is NaN, or an infinity among those of the values, is the result of every row that sees its key, whichever kernel the number
    of rows takes; the other rows have their bits.  A key before the tree, and a node."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = made = make(torch, D, [new], [total], 4, 2, 128, 16, bits, seed=4)
    seen = trees(np.random.default_rng(new), [new])
    words = words_of(seen)
    clean = run(torch, D, *made, words)
    check(clean, made, seen)
    parts = [()] if bits == 8 else [(0,), (1,)]
    for at in (total - new - 20, total - new + new // 2):
        page, off = int(table[0, at // 16]), at % 16
        sees = seen[0][:, at - (total - new)] if at >= total - new else np.ones(new, bool)
        assert sees.any()
        for step, odd in ((cache.k_step, float("nan")), (cache.v_step, float("nan")), (cache.v_step, float("inf")), (cache.v_step, float("-inf"))):
            for part in parts:
                keep = step[(page, 1, off, *part)].clone()
                step[(page, 1, off, *part)] = odd
                got = run(torch, D, *made, words)
                step[(page, 1, off, *part)] = keep
                assert np.array_equal(got[~sees], clean[~sees]) and np.array_equal(got[:, :2], clean[:, :2])
                assert not np.isfinite(got[sees][:, 2:]).any(), (at, odd, part)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [2, 100])
@pytest.mark.parametrize("scale", [0.0, -0.25])
def test_scales_of_zero_and_below(scale, new, bits):
    import torch
    from paper_2507_12205_amd import device as D
    made = make(torch, D, [new, 1], [400, 1], 2, 2, 64, 16, bits, seed=13)
    seen = trees(np.random.default_rng(2), [new, 1])
    check(run(torch, D, *made, words_of(seen), scale=scale), made, seen, scale)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,total", [(6, 333), (40, 200), (200, 330), (100, 3000)])
def test_values_of_very_different_sizes(new, total, bits):
    """Rows of zeros and of equal values, which have no step, beside steps that are eight powers of ten apart.

    The bound is that above with p times a key's own largest value in the place of the largest of all: weights go to the products with their step, below
    the normal range by 2^-25 of the largest such product, and codes are 127 at most; in 4 bits a row's code 8 is at most 8/15 of its range
    away from any of its values, 16/15 of its largest."""
    import torch
    from paper_2507_12205_amd import device as D
    rng = np.random.default_rng(new)
    made = make(torch, D, [new], [total], 4, 2, 128, 16, bits, seed=31, stale=float("nan"))
    cache, q, start, lens, table = made
    shape = (total, 2, 128)
    k = rng.normal(size=shape)
    v = rng.normal(size=shape) * rng.choice([0.0, 1e-6, 1e-3, 1.0, 1e4], size=(total, 2, 1))
    v[rng.random((total, 2)) < 0.1] = 0.75
    i = np.arange(total)
    slots = torch.from_numpy(table[0, i // 16].astype(np.int64) * 16 + i % 16).cuda()
    D.kv_write(cache, *(torch.from_numpy(x.astype(np.float16)).cuda() for x in (k, v)), slots)
    seen = trees(rng, [new])
    got = run(torch, D, *made, words_of(seen))
    keys, vals = values(cache)
    q64 = q.cpu().numpy().astype(np.float64)
    want, size = tree.attention(q64, keys, vals, start, lens, table, seen, 128 ** -0.5)
    reach = np.broadcast_to(np.abs(vals).max(-1, keepdims=True), vals.shape)
    most, _ = tree.attention(q64, keys, reach, start, lens, table, seen, 128 ** -0.5)
    bound = 2 ** -11 * np.abs(want) + (2 ** -11 + 2 ** -14) * (size + (16 / 15 * most if bits == 4 else 0.0)) + total * 2 ** -24 * most + 2 ** -25
    assert np.isfinite(got).all() and (np.abs(got - want) <= bound).all()
    zero = torch.zeros(shape, dtype=torch.float16, device="cuda")
    D.kv_write(cache, torch.from_numpy(k.astype(np.float16)).cuda(), zero, slots)
    assert not run(torch, D, *made, words_of(seen)).any()
    D.kv_write(cache, torch.from_numpy(k.astype(np.float16)).cuda(), zero + 0.75, slots)
    # of equal values the mean is that value: in 4 bits kept as it is, in 8 as 127 steps of it
    assert (np.abs(run(torch, D, *made, words_of(seen)) - 0.75) <= 0.75 * (2 ** -11 + 2 ** -14 + (2 ** -11 if bits == 8 else 0))).all()


@pytest.mark.parametrize("new,heads,kv_heads,dim", [(5, 4, 1, 128), (33, 6, 6, 64), (64, 4, 4, 128), (16, 8, 2, 96), (9, 6, 2, 32)])
@pytest.mark.parametrize("past", [1, 4, 40, 1500])
def test_weights_of_up_to_64_rows(past, new, heads, kv_heads, dim):
    """FP16, 17 to 64 rows of a head of the cache: a weight is two FP16 values, 2^-22 of it off and of the range below the normal one 2^-25 of the largest.  The
    result is rounded to FP16 (2^-11 of it, 2^-25), scores are off by 2^-22 of scale times sum |q| times the largest |k| (sums of dim products), which the
    weight has twice, and 2^-14 covers sums and exponentials, as in test_gpu_attention_codes."""
    import torch
    from paper_2507_12205_amd import device as D
    rng, batch = np.random.default_rng(past + new), 6
    cache, q, start, lens, table = made = make(torch, D, [new] * batch, [past + new] * batch, heads, kv_heads, dim, 16, 16, seed=past, stale=float("nan"))
    seen = trees(rng, [new] * batch)
    got = run(torch, D, *made, words_of(seen))
    (k, v), x = values(cache), q.cpu().numpy().astype(np.float64)
    want, size = tree.attention(x, k, v, start, lens, table, seen, dim ** -0.5)
    keys = max(np.abs(ref.gather(k, table[b], n)).max() for b, n in enumerate(lens))
    top = max(np.abs(ref.gather(v, table[b], n)).max() for b, n in enumerate(lens))
    score = 2.0 ** -22 * dim ** -0.5 * np.abs(x).sum(-1, keepdims=True) * keys
    bound = 2 ** -11 * np.abs(want) + (2 ** -22 + 2 ** -14 + 2 * score) * size + (past + new) * 2 ** -24 * top + 2 ** -25
    worst = np.max(np.abs(got - want) / bound)
    assert worst <= 1.0, worst


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new,total", [([4, 1], [2500, 900]), ([50, 70], [2500, 900])])
def test_the_same_bits_every_time(new, total, bits):
    import torch
    from paper_2507_12205_amd import device as D
    made = make(torch, D, new, total, 8, 2, 128, 16, bits, seed=5)
    words = words_of(trees(np.random.default_rng(2), new))
    first = run(torch, D, *made, words)
    for _ in range(3):
        assert np.array_equal(run(torch, D, *made, words), first)
    assert np.array_equal(run(torch, D, *made, words, workspace=None), first)


@pytest.mark.parametrize("bits", [16, 4])
def test_tokens_beyond_max_new(bits):
    """More tokens of a sequence than max_new: the first max_new are as they are, where they see none of the others (whose words there are none of)."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, total, table = made = make(torch, D, [40, 90], [200, 300], 4, 2, 64, 16, bits, seed=5)
    seen = trees(np.random.default_rng(2), [40, 90])
    full = run(torch, D, *made, words_of(seen))
    short = run(torch, D, *made, np.ascontiguousarray(words_of(seen)[:, :2]), max_new=64)
    k, v = values(cache)
    assert np.isfinite(short[:40]).all() and np.abs(short[:104] - full[:104]).max() <= 2 ** -9 * np.abs(v).max()


def test_tree_seen():
    import torch
    from paper_2507_12205_amd import device as D
    rng = np.random.default_rng(3)
    parents = [tree.parents(rng, n) for n in (1, 70, 33)]
    assert np.array_equal(D.tree_seen(parents).cpu().numpy(), words_of([tree.tree_seen(p) for p in parents]))
    assert D.tree_seen([]).shape == (0, 1)
    with pytest.raises(ValueError):
        D.tree_seen([[-1, 1]])
    torch.cuda.synchronize()


def test_in_a_graph_and_on_another_stream():
    """Lengths and masks are read when the kernels run: a captured step goes on with what the tensors hold then."""
    import torch
    from paper_2507_12205_amd import device as D
    for new, total in (([5], [600]), ([70], [600])):
        made = cache, q, start, lens, table = make(torch, D, new, total, 4, 2, 64, 16, 8, seed=6)
        s, n, t = (torch.from_numpy(x).cuda() for x in (start, lens, table))
        words = torch.zeros((new[0], 3), dtype=torch.int32, device="cuda")
        out, eager = torch.empty_like(q), torch.empty_like(q)
        ws = D.attention_workspace(cache, q, 1, new[0], table.shape[1] * 16)
        side = torch.cuda.Stream()
        D.attention_tree(cache, q, out, s, n, t, words, new[0], None, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            D.attention_tree(cache, q, out, s, n, t, words, new[0], None, ws)
        for turn, length in enumerate((600, 599, 90, 70, 3, 0, 600)):
            seen = trees(np.random.default_rng(turn), new)
            w = words_of(seen)
            words.zero_()
            words[:, :w.shape[1]] = torch.from_numpy(w).cuda()
            n.fill_(length)
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            check(out.cpu().numpy().astype(np.float64), (cache, q, start, np.array([length], np.int32), table), seen)
            D.attention_tree(cache, q, eager, s, n, t, words, new[0], None, None, stream=side)
            side.synchronize()
            assert torch.equal(eager, out)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new,total", [([7, 0, 5], [1000, 30, 40]), ([40, 70], [900, 2000]), ([3, 2] * 40, [600, 20] * 40)])
def test_rows_of_no_sequence_stay(new, total, bits):
    """Tokens before the first sequence and behind the last one are left as they were, and change nothing."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = made = make(torch, D, new, total, 4, 2, 64, 16, bits, seed=8)
    words = words_of(trees(np.random.default_rng(1), new))
    want = run(torch, D, *made, words)
    wide = torch.randn((len(q) + 9, *q.shape[1:]), device="cuda").half()
    wide[4:4 + len(q)] = q
    out = torch.full_like(wide, 77.0)
    seen = np.full((len(wide), words.shape[1]), -1, np.int32)
    seen[4:4 + len(q)] = words
    args = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (start + 4, lens, table, seen)]
    D.attention_tree(cache, wide, out, *args, int(np.diff(start).max()))
    got = out.cpu().numpy().astype(np.float64)
    assert (got[:4] == 77).all() and (got[4 + len(q):] == 77).all()
    v = values(cache)[1]
    assert np.abs(got[4:4 + len(q)] - want).max() <= 2 ** -9 * np.abs(v).max()          # (splits may differ with the number of tokens)


def test_very_many_sequences():
    """More sequences than a grid's second dimension holds of workgroups at once: each has one key, which is the result."""
    import torch
    from paper_2507_12205_amd import device as D
    n = 40000
    cache = D.kv_cache(n, 1, 16, 16)
    k, v, q = (torch.randn((n, 1, 16), device="cuda").half() for _ in range(3))
    D.kv_write(cache, k, v, torch.arange(n, device="cuda") * 16)
    out, i = torch.full_like(q, float("nan")), torch.arange(n + 1, dtype=torch.int32, device="cuda")
    D.attention_tree(cache, q, out, i, torch.ones(n, dtype=torch.int32, device="cuda"), i[:n, None], torch.ones((n, 1), dtype=torch.int32, device="cuda"), 1)
    assert torch.equal(out, v)


@pytest.mark.parametrize("bits", [16, 8])
def test_two_graphs_that_share_a_workspace(bits):
    """Attention of a row of new tokens and of trees, captured apart with one workspace for both: its contents do not matter before and after."""
    import torch
    from paper_2507_12205_amd import device as D
    made = [make(torch, D, new, total, 4, 2, 64, 16, bits, seed=i) for i, (new, total) in enumerate((([5, 2], [1600, 700]), ([40, 9, 3], [900, 2000, 30])))]
    seen = [trees(np.random.default_rng(i), list(np.diff(m[2]))) for i, m in enumerate(made)]
    ws = torch.empty(max(D.attention_workspace(m[0], m[1], len(m[3]), 40, 2048).nbytes for m in made), dtype=torch.uint8, device="cuda")
    graphs, outs, eager, kept = [], [], [], []
    for m, s in zip(made, seen):
        cache, q, *rest = m
        args = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (*rest, words_of(s))]
        tree_out, row_out, most = torch.empty_like(q), torch.empty_like(q), int(np.diff(m[2]).max())
        kept.append(args)                                    # what the graphs read

        def call(work):
            D.attention_tree(cache, q, tree_out, *args, most, None, work)
            D.attention(cache, q, row_out, *args[:3], most, None, work)
        call(None)
        eager.append((tree_out.clone(), row_out.clone()))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(ws)
        graphs.append(graph)
        outs.append((tree_out, row_out))
    for turn in (0, 1, 1, 0, 1, 0, 0):
        for t in outs[turn]:
            t.fill_(float("nan"))
        graphs[turn].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs[turn], eager[turn]))
        if turn:
            ws.fill_(255)
