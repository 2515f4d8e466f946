"""Attention over the paged cache against 64 bits: lengths, heads, widths, layouts, what lies in masked places.

The bound: the result is rounded to FP16 (2^-11 of it), so are the weights (2^-11 of the sum of p |v|; those below the normal range by 2^-25
each, of the largest |v|); sums, exponentials and scores in FP32 come to far less than the 2^-14 allowed for them."""
import numpy as np
import pytest
import serve_reference as ref

pytestmark = pytest.mark.gpu


def make(torch, D, new, total, heads, kv_heads, dim, page, bits, seed=0, layout="tokens", stale=None):
    """A cache written by kv_write, whose other places hold `stale`, and the new tokens' q."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in total]
    pages = sum(need) + 2
    cache = D.kv_cache(pages, kv_heads, page, dim, bits)
    for t in (cache.k, cache.v, cache.k_step, cache.v_step):
        if t is not None and stale is not None:
            t.fill_(stale if t.dtype.is_floating_point else 77)
    order, at = rng.permutation(pages), 0
    width = max(need + [0]) + 1
    table = np.full((len(total), width), -7, np.int32)          # what is beyond a sequence's pages is not looked at
    for b, n in enumerate(total):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        if n:
            i = np.arange(n)
            slots = torch.from_numpy((table[b, i // page].astype(np.int64) * page + i % page)).cuda()
            k, v = (torch.from_numpy(rng.normal(size=(n, kv_heads, dim)).astype(np.float16)).cuda() for _ in range(2))
            D.kv_write(cache, k, v, slots)
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = torch.from_numpy((2 * rng.normal(size=(int(start[-1]), heads, dim))).astype(np.float16)).cuda()
    return cache, q, start, np.asarray(total, np.int32), table


def values(cache):
    k, v = ((None if t is None else t.cpu().numpy()) for t in (cache.k, cache.v))
    ks, vs = ((None if t is None else t.cpu().numpy()) for t in (cache.k_step, cache.v_step))
    return ref.decode(k, ks, cache.bits), ref.decode(v, vs, cache.bits)


def place(x, layout, torch):
    t, h, d = x.shape
    if layout == "columns":
        return x.permute(1, 2, 0).contiguous().permute(2, 0, 1)
    if layout == "odd":
        wide = torch.zeros((t, h, d + 3), dtype=x.dtype, device=x.device)
        wide[:, :, 1:d + 1] = x
        return wide[:, :, 1:d + 1]
    if layout == "heads":
        return x.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    return x


def run(torch, D, cache, q, start, total, table, layout="tokens", scale=None, max_new=None, workspace="own"):
    new = np.diff(start)
    out = place(torch.full_like(q, float("nan")), layout, torch)
    args = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (start, total, table)]
    most = int(new.max()) if max_new is None else max_new
    ws = D.attention_workspace(cache, q, len(total), most, table.shape[1] * cache.page_size) if workspace == "own" else workspace
    if ws is not None and ws.numel():
        ws.fill_(255)                                        # NaN all over: nothing is read that was not written
    D.attention(cache, place(q, layout, torch), out, *args, most, scale, ws)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64)


def check(got, cache, q, start, total, table, scale=None):
    k, v = values(cache)
    scale = cache.head_dim ** -0.5 if scale is None else scale
    want, size = ref.attention(q.cpu().numpy().astype(np.float64), k, v, start, total, table, scale)
    assert np.isfinite(got).all()
    top = max((np.abs(ref.gather(v, table[b], n)).max() for b, n in enumerate(total) if n), default=0.0)
    # (4-bit codes are taken from the middle of their range: eight steps at most, a row's whole reach of 15 below twice its largest value)
    bound = 2 ** -11 * np.abs(want) + (2 ** -11 + 2 ** -14) * (size + (top if cache.bits == 4 else 0.0)) + max(total) * 2 ** -24 * top + 2 ** -25
    worst = np.max(np.abs(got - want) / bound) if got.size else 0.0
    assert worst <= 1.0, worst


CASES = [
    # new tokens and keys of each sequence, heads, heads of the cache, dim, page
    ([1], [1], 1, 1, 16, 16), ([1], [33], 4, 2, 64, 16), ([1, 1, 1], [5, 300, 64], 12, 12, 64, 16), ([1], [2049], 8, 1, 128, 64),
    ([8], [1000], 4, 4, 128, 32), ([3, 1, 7, 2], [3, 17, 260, 513], 8, 2, 128, 16), ([17, 40], [17, 333], 6, 2, 80, 32),
    ([130], [130], 2, 1, 96, 16), ([65, 1, 33], [700, 1, 33], 4, 4, 64, 128), ([5], [4100], 2, 2, 256, 256), ([200], [456], 3, 3, 128, 64),
    ([1, 2], [100, 31], 16, 1, 240, 16), ([70], [70], 5, 5, 48, 1024),
]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("case", CASES)
def test_against_64_bits(case, bits):
    import torch
    from paper_2507_12205_amd import device as D
    made = make(torch, D, *case, bits, seed=len(CASES) * bits + CASES.index(case), stale=float("nan"))
    check(run(torch, D, *made), *made)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("layout", ["columns", "odd", "heads"])
@pytest.mark.parametrize("new,total", [([8], [300]), ([150, 3], [150, 90])])
def test_layouts(layout, bits, new, total):
    import torch
    from paper_2507_12205_amd import device as D
    made = make(torch, D, new, total, 8, 4, 128, 32, bits, seed=3, stale=float("inf"))
    assert np.array_equal(run(torch, D, *made, layout=layout), run(torch, D, *made))


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_rows_that_see_nothing(bits):
    """More new tokens than keys: the first ones see none and get zeros; sequences without tokens, and without keys."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, total, table = make(torch, D, [5, 0, 2, 40], [3, 20, 0, 30], 4, 2, 64, 16, bits, seed=9, stale=float("nan"))
    got = run(torch, D, cache, q, start, total, table)
    assert not got[:2].any() and not got[5:7].any() and not got[7:17].any()
    check(got, cache, q, start, total, table)


@pytest.mark.parametrize("new,total", [(6, 70), (40, 200), (200, 330), (6, 3000)])
@pytest.mark.parametrize("odd", [float("nan"), float("inf")])
def test_values_that_later_tokens_only_see(new, total, odd):
    """An infinity or NaN in a token's key or value stays with the tokens that see it."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, lens, table = make(torch, D, [new], [total], 4, 2, 128, 16, 16, seed=4)
    clean = run(torch, D, cache, q, start, lens, table)
    at = total - new // 2                                    # a new token in the middle of the chunk
    page, off = int(table[0, at // 16]), at % 16
    first = at - (total - new)
    for tensor in (cache.v, cache.k):
        keep = tensor[page, 1, off, 5].clone()
        tensor[page, 1, off, 5] = odd
        got = run(torch, D, cache, q, start, lens, table)
        assert np.array_equal(got[:first], clean[:first]) and np.array_equal(got[:, :2], clean[:, :2])
        assert not np.isfinite(got[first:, 2:, 5] if tensor is cache.v else got[first:, 2:]).any() or odd == float("inf")
        if tensor is cache.v:
            rest = [d for d in range(128) if d != 5]
            assert np.allclose(got[:, :, rest], clean[:, :, rest], rtol=2 ** -9, atol=2 ** -12)
            assert not np.isfinite(got[first:, 2:, 5]).any()
        tensor[page, 1, off, 5] = keep


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [2, 100])
def test_scores_far_apart(new, bits):
    """Softmax with scores in the hundreds: the running maximum moves by more than FP32's exponents hold; the scale is the caller's."""
    import torch
    from paper_2507_12205_amd import device as D
    made = make(torch, D, [new], [400], 2, 2, 64, 16, bits, seed=12)
    k, v = values(made[0])
    got = run(torch, D, *made, scale=4.0)
    want, size = ref.attention(made[1].cpu().numpy().astype(np.float64), k, v, *made[2:], 4.0)
    # scores of up to some 500 in FP32: their own rounding (2^-23 of the sum of |q k|, 4 * 64 * 10 at most) moves p by up to 2^-11
    top = np.abs(v).max()
    assert (np.abs(got - want) <= 2 ** -11 * np.abs(want) + 3 * 2 ** -11 * (size + top)).all()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [2, 100])
@pytest.mark.parametrize("scale", [0.0, -0.25])
def test_scales_of_zero_and_below(scale, new, bits):
    """0: the mean of the values that a row sees, and of no other."""
    import torch
    from paper_2507_12205_amd import device as D
    made = make(torch, D, [new, 1], [400, 1], 2, 2, 64, 16, bits, seed=13)
    check(run(torch, D, *made, scale=scale), *made, scale=scale)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_the_same_bits_every_time(bits):
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, total, table = make(torch, D, [4, 1], [2500, 900], 8, 2, 128, 16, bits, seed=5)
    first = run(torch, D, cache, q, start, total, table)
    for _ in range(3):
        assert np.array_equal(run(torch, D, cache, q, start, total, table), first)
    assert np.array_equal(run(torch, D, cache, q, start, total, table, workspace=None), first)
    wide = np.full((2, 3 * table.shape[1]), 2 ** 31 - 1, np.int32)          # places that hold no page at all
    wide[:, :table.shape[1]] = table
    check(run(torch, D, cache, q, start, total, wide), cache, q, start, total, wide)


def test_in_a_graph_and_on_another_stream():
    """Lengths and places are read when the kernels run: a captured step goes on with what the tensors hold then."""
    import torch
    from paper_2507_12205_amd import device as D
    cache, q, start, total, table = make(torch, D, [2], [600], 4, 2, 64, 16, 8, seed=6)
    s, n, t = (torch.from_numpy(x).cuda() for x in (start, total, table))
    out = torch.empty_like(q)
    ws = D.attention_workspace(cache, q, 1, 2, table.shape[1] * 16)
    k, v = torch.randn(2, 2, 64, device="cuda").half(), torch.randn(2, 2, 64, device="cuda").half()
    slots = torch.tensor([int(table[0, 37]) * 16 + 6, int(table[0, 37]) * 16 + 7], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        D.kv_write(cache, k, v, slots)
        D.attention(cache, q, out, s, n, t, 2, None, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.kv_write(cache, k, v, slots)
        D.attention(cache, q, out, s, n, t, 2, None, ws)
    for length in (600, 599, 40, 1, 0, 600):
        n.fill_(length)
        k.normal_()
        v.normal_()
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().numpy().astype(np.float64)
        check(got, cache, q, start, np.array([length], np.int32), table)
        eager = torch.empty_like(out)
        D.attention(cache, q, eager, s, n, t, 2, None, None, stream=side)
        side.synchronize()
        assert torch.equal(eager, out)
