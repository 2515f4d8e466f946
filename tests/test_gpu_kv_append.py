"""Keys and values into the paged cache with the rotation by position on the way: what is written and what comes out in q_out, against the
definition in 64 bits.

Bounds.  A rotated value is a cos t - b sin t with cos and sin rounded to FP32 (2^-24 each of |a|, |b|), products and sum in FP32 (three roundings of at
most |a| + |b|): 4 * 2^-24 (|a| + |b|); the angle of position n is off by n * 2^-51 at most (a product in 64 bits, taken to turns).  Rounded once:
to FP16 (2^-11 of it, 2^-25 where that is less), or to a code: half a step; with 4 bits the lowest value is rounded to FP16 (2^-11 of it) and so is the
step (the last code ends up to 15 * 2^-11 steps, or 15 * 2^-25, from the largest value)."""
import numpy as np
import pytest
import serve_reference as ref
import tree_reference as tree
from test_gpu_kv_cache import layout, values

pytestmark = pytest.mark.gpu

# tokens, heads of q, heads of the cache, dim, rotary, page
SHAPES = [(1, 1, 1, 16, 16, 16), (7, 6, 3, 80, 80, 16), (64, 12, 12, 64, 32, 32), (33, 4, 2, 256, 256, 64), (130, 16, 8, 128, 128, 256),
          (5, 2, 1, 240, 2, 1024), (21, 4, 4, 80, 20, 16), (40, 0, 2, 128, 96, 32), (3, 5, 5, 48, 46, 16), (17, 2, 2, 64, 0, 16)]


def frequencies(pairs):
    return 10000.0 ** (-np.arange(pairs) / max(pairs, 1))


def rotation_error(x, position, frequency, neighbours):
    """The most that a rotated value can be off before it is rounded."""
    x = np.abs(np.asarray(x, np.float64))
    pairs, both = len(frequency), np.zeros(x.shape)
    if neighbours:
        both[..., 0:2 * pairs:2] = both[..., 1:2 * pairs:2] = x[..., 0:2 * pairs:2] + x[..., 1:2 * pairs:2]
    else:
        both[..., :pairs] = both[..., pairs:2 * pairs] = x[..., :pairs] + x[..., pairs:2 * pairs]
    return (4 * 2.0 ** -24 + np.abs(position.astype(np.float64))[:, None, None] * 2.0 ** -51) * both


def near_halves(got, want, error):
    assert (np.abs(got - want) <= error + 2.0 ** -11 * (np.abs(want) + error) + 2.0 ** -25).all()


def near_codes(got, want, error, bits):
    """Rows of values as the cache holds them."""
    low, reach = want.min(-1, keepdims=True), np.abs(want).max(-1, keepdims=True)
    error = error.max(-1, keepdims=True)
    if bits == 8:
        step = (reach + error) / 127
        slack = 0.5 * step
    else:
        step = (want.max(-1, keepdims=True) - low + 2 * error + 2.0 ** -11 * np.abs(low) + 2.0 ** -25) / 15 * (1 + 2.0 ** -11) + 2.0 ** -25
        slack = 0.5 * step + 2.0 ** -11 * np.abs(low) + 2.0 ** -25 + 15 * (2.0 ** -11 * step + 2.0 ** -25)
    assert (np.abs(got - want) <= slack + error + 2.0 ** -20 * reach).all()


def cached(cache, slots, torch):
    """(tokens, heads, dim) of k and v as the cache holds them."""
    out = []
    for code, step in ((cache.k, cache.k_step), (cache.v, cache.v_step)):
        x = ref.decode(code.cpu().numpy(), None if step is None else step.cpu().numpy(), cache.bits)
        out.append(x[slots // cache.page_size, :, slots % cache.page_size])
    return out


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("kind", ["plain", "columns", "heads", "odd"])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_64_bits(shape, kind, neighbours, bits):
    import torch
    from paper_2507_12205_amd import device as D
    tokens, q_heads, heads, dim, rotary, page = shape
    rng = np.random.default_rng(tokens)
    pages = 2 * (-(-tokens // page)) + 1
    cache = D.kv_cache(pages, heads, page, dim, bits)
    every = [t for t in (cache.k, cache.v, cache.k_step, cache.v_step) if t is not None]
    for t in every:
        t.fill_(3)
    k, v = values((tokens, heads, dim), 1, torch), values((tokens, heads, dim), 5, torch)
    q = values((tokens, q_heads, dim), 7, torch) if q_heads else None
    k[0, 0] = 0                                              # a row of zeros
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    if tokens > 6:
        slots[2], slots[5] = -1, pages * page
    position = rng.integers(0, 1 << rng.integers(1, 21, tokens)).astype(np.int32)
    position[-1] = 2 ** 31 - 1
    if tokens > 1:
        position[0] = -5
    freq = frequencies(rotary // 2)
    before = [t.clone() for t in every]
    args = [torch.from_numpy(x).cuda() for x in (slots, position, freq)]
    q_out = None if q is None else layout(torch.full_like(q, float("nan")), kind, torch)
    got = D.kv_append(cache, layout(k, kind, torch), layout(v, kind, torch), *args, None if q is None else layout(q, kind, torch), q_out, neighbours)
    torch.cuda.synchronize()
    assert got is q_out
    if q is not None:
        x = q.cpu().numpy()
        near_halves(q_out.cpu().numpy().astype(np.float64), tree.rotate(x, position, freq, neighbours), rotation_error(x, position, freq, neighbours))
    valid = (slots >= 0) & (slots < pages * page)
    kx, vx = k.cpu().numpy()[valid], v.cpu().numpy()[valid]
    kc, vc = cached(cache, slots[valid], torch)
    want, error = tree.rotate(kx, position[valid], freq, neighbours), rotation_error(kx, position[valid], freq, neighbours)
    if bits == 16:
        near_halves(kc, want, error)
        assert np.array_equal(vc, vx.astype(np.float64))
    else:
        near_codes(kc, want, error, bits)
        near_codes(vc, vx.astype(np.float64), np.zeros(vx.shape), bits)
    free = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    free[torch.from_numpy(slots[valid]).cuda()] = False
    free = free.view(pages, page)
    for now, was in zip(every, before):
        assert torch.equal(now.transpose(1, 2)[free], was.transpose(1, 2)[free])


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("tokens", [9, 16, 24, 72, 200, 328])
@pytest.mark.parametrize("q_heads,heads,dim,rotary,neighbours", [(6, 3, 64, 64, False), (3, 5, 128, 64, True), (2, 1, 80, 36, False), (9, 2, 256, 256, False),
                                                                 (1, 3, 16, 16, True), (0, 2, 240, 100, False), (20, 1, 32, 32, False)])
def test_columns_give_the_same_bits(q_heads, heads, dim, rotary, neighbours, tokens, bits):
    """Columns that start at multiples of 16 bytes and that do not, each of the tensors in them or not, tokens that are no multiple of 16: what rows give; and
    nothing is written beside the tokens."""
    import torch
    from paper_2507_12205_amd import device as D
    x = [values((tokens, n, dim), 3 + i, torch) for i, n in enumerate((heads, heads, q_heads))]
    slots = torch.randperm(16 * 30, device="cuda")[:tokens]
    position = torch.arange(tokens, dtype=torch.int32, device="cuda") * 1000
    frequency = D.rotary_frequency(rotary // 2)

    def wide(t, columns, pad):
        """The tensor itself, or tokens after one another in columns of ceil8(tokens) + pad places, and all those places."""
        if not columns:
            return t, t
        every = torch.full((t.shape[1], dim, -(-tokens // 8) * 8 + pad), 7.0, dtype=t.dtype, device=t.device)
        every[:, :, :tokens] = t.permute(1, 2, 0)
        return every[:, :, :tokens].permute(2, 0, 1), every

    def run(columns, pad=0, in_place=False):
        cache = D.kv_cache(30, heads, 16, dim, bits)
        (k, _), (v, _), (q, all_q) = (wide(t.clone(), c, pad) for t, c in zip(x, columns))
        out, all_out = (q, all_q) if in_place else wide(torch.zeros_like(x[2]), columns[3], pad)
        D.kv_append(cache, k, v, slots, position, frequency, *((q, out) if q_heads else ()), neighbours=neighbours)
        if q_heads and out is not x[2] and all_out.shape[-1] > tokens and all_out.dim() == 3 and all_out.shape[1] == dim:
            assert (all_out[:, :, tokens:] == 7.0).all()
        return [t for t in (cache.k, cache.v, cache.k_step, cache.v_step, out if q_heads else None) if t is not None]

    want = run((False,) * 4)
    for case in ([(True,) * 4], [(True,) * 4, 1], [(True,) * 4, 8, True], [(True, True, False, True)], [(False, False, True, False)], [(True, False, True, True), 8]):
        assert all(torch.equal(a, b) for a, b in zip(run(*case), want)), case


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rotary", [0, 64])
def test_without_a_turn_it_is_kv_write(rotary, bits):
    """No pairs, or position 0: bit for bit what kv_write leaves, and q as it was."""
    import torch
    from paper_2507_12205_amd import device as D
    a, b = (D.kv_cache(9, 3, 16, 64, bits) for _ in range(2))
    k, v, q = values((100, 3, 64), 2, torch), values((100, 3, 64), 3, torch), values((100, 9, 64), 4, torch)
    slots = torch.randperm(144, device="cuda")[:100]
    D.kv_write(a, k, v, slots)
    out = D.kv_append(b, k, v, slots, torch.zeros(100, dtype=torch.int32, device="cuda"), D.rotary_frequency(rotary // 2), q, torch.empty_like(q))
    for x, y in zip((a.k, a.v, a.k_step, a.v_step), (b.k, b.v, b.k_step, b.v_step)):
        assert x is None or torch.equal(x, y)
    assert torch.equal(out, q)


@pytest.mark.parametrize("rotary,neighbours", [(0, False), (16, False), (16, True), (10, False)])
def test_without_a_turn_it_is_kv_write_in_4_bits(rotary, neighbours):
    """The step is the range divided by 15 in FP32 and then rounded to FP16; of keys that are rotated, if by nothing, the range times 1/15.  Rows whose range is
    15 times the middle of two FP16 values, for which the two differ in 439 of 1024 cases, and random ones."""
    import torch
    from paper_2507_12205_amd import device as D
    n, rng = 4096, np.random.default_rng(1)
    a, b = (D.kv_cache(n // 16, 4, 16, 16, 4) for _ in range(2))
    x = rng.normal(size=(2, n, 4, 16)) * rng.choice([1e-3, 1.0, 30.0], size=(2, n, 4, 1))
    spread = 15 * (2 * np.arange(1024, 2048) + 1)            # 16 bits: the ten upper ones above zero, the six lower ones below
    high, low = (spread >> 6 << 6) * 2.0 ** -14, -(spread & 63) * 2.0 ** -14
    ties = low[:, None, None] + (high - low)[:, None, None] * rng.random((1024, 4, 16))
    ties[..., 3], ties[..., 11] = low[:, None], high[:, None]
    x[0, :1024], x[1, 1024:2048] = ties, ties
    k, v = (torch.from_numpy(t.astype(np.float16)).cuda() for t in x)
    assert (k[:1024].float().amax(-1) - k[:1024].float().amin(-1) == torch.from_numpy(spread * 2.0 ** -14).cuda()[:, None]).all()
    slots = torch.randperm(n, device="cuda")
    D.kv_write(a, k, v, slots)
    D.kv_append(b, k, v, slots, torch.zeros(n, dtype=torch.int32, device="cuda"), D.rotary_frequency(rotary // 2), neighbours=neighbours)
    assert torch.equal(a.v, b.v) and torch.equal(a.v_step, b.v_step)
    if rotary == 0:
        assert torch.equal(a.k, b.k) and torch.equal(a.k_step, b.k_step)
    else:
        low, high = k.float().amin(-1), k.float().amax(-1)
        step = ((high - low) * torch.tensor(1 / 15, device="cuda")).half()
        want = torch.stack([step, low.half()], -1)[slots.argsort()].view(n // 16, 16, 4, 2).transpose(1, 2)
        assert torch.equal(b.k_step, want)
        apart = (a.k_step[..., 0].view(torch.int16) - b.k_step[..., 0].view(torch.int16)).abs()          # neighbouring FP16 values
        assert apart.max() == 1 and torch.equal(a.k_step[..., 1], b.k_step[..., 1])


@pytest.mark.parametrize("rotary,neighbours", [(64, False), (64, True), (20, False), (62, False)])
@pytest.mark.parametrize("kind", ["plain", "columns"])
def test_queries_in_place(kind, rotary, neighbours):
    import torch
    from paper_2507_12205_amd import device as D
    cache = D.kv_cache(20, 2, 16, 64, 8)
    k, q = values((200, 2, 64), 2, torch), layout(values((200, 6, 64), 4, torch), kind, torch)
    slots, position = torch.arange(200, device="cuda"), torch.arange(1000, 1200, dtype=torch.int32, device="cuda")
    freq = D.rotary_frequency(rotary // 2, 500000.0)
    apart = D.kv_append(cache, k, k, slots, position, freq, q, torch.empty_like(q), neighbours)
    assert D.kv_append(cache, k, k, slots, position, freq, q, None, neighbours) is q
    assert torch.equal(q, apart)


@pytest.mark.parametrize("bits", [8, 4])
def test_values_that_are_not_finite(bits):
    """NaN counts as 0 and what is beyond FP16's largest value as that: every code stands for a finite value."""
    import torch
    from paper_2507_12205_amd import device as D
    cache = D.kv_cache(1, 1, 16, 32, bits)
    x = torch.randn(5, 1, 32, dtype=torch.float16, device="cuda")
    x[0, 0, 3], x[1, 0, 4], x[2, 0, 5], x[3, 0], x[4, 0] = float("nan"), float("inf"), float("-inf"), float("nan"), 65504.0
    slots = torch.arange(5, device="cuda")
    D.kv_append(cache, x, x, slots, torch.full((5,), 3, dtype=torch.int32, device="cuda"), D.rotary_frequency(16))
    k, v = torch.empty_like(x), torch.empty_like(x)
    D.kv_read(cache, slots, k, v)
    assert torch.isfinite(k).all() and torch.isfinite(v).all() and not k[3].any()


def test_rows_that_are_not_finite_stay_rows():
    """16 bits: NaN and infinities as arithmetic makes them, in their pair and nowhere else."""
    import torch
    from paper_2507_12205_amd import device as D
    cache = D.kv_cache(1, 1, 16, 64, 16)
    x = torch.randn(2, 1, 64, dtype=torch.float16, device="cuda")
    clean = x.clone()
    x[0, 0, 3], x[1, 0, 60] = float("nan"), float("inf")
    out = []
    for t in (clean, x):
        D.kv_append(cache, t, t, torch.arange(2, device="cuda"), torch.full((2,), 3, dtype=torch.int32, device="cuda"), D.rotary_frequency(16))
        out.append(cache.k[0, 0, :2].clone())
    same = out[0] == out[1]
    assert [i for i in range(64) if not same[0, i]] == [3, 19] and [i for i in range(64) if not same[1, i]] == [60]


def test_a_position_far_off():
    """Angles go by 64 bits: position 2^30 and a frequency whose multiple of it is a whole number of turns give the key itself."""
    import torch
    from paper_2507_12205_amd import device as D
    cache = D.kv_cache(1, 1, 16, 32, 16)
    x = torch.randn(1, 1, 32, dtype=torch.float16, device="cuda")
    freq = torch.full((16,), 2 * np.pi / 1024, dtype=torch.float64, device="cuda")
    D.kv_append(cache, x, x, torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 1 << 30, dtype=torch.int32, device="cuda"), freq)
    # 2 pi / 1024 is rounded by up to 2^-54 of itself: the angle is off by up to 2^30 * 2^-7 * 2^-53 < 2^-29
    near_halves(cache.k[0, 0, 0].double().cpu().numpy(), x[0, 0].double().cpu().numpy(), 4 * 2.0 ** -24 * np.full(32, 10.0))


@pytest.mark.parametrize("tokens", [3, 100])
def test_in_a_graph_and_on_another_stream(tokens):
    """Positions and places are read when the kernel runs."""
    import torch
    from paper_2507_12205_amd import device as D
    a, b = (D.kv_cache(16, 2, 16, 64, 8) for _ in range(2))
    k, v, q = values((tokens, 2, 64), 2, torch), values((tokens, 2, 64), 3, torch), values((tokens, 4, 64), 4, torch)
    slots, position = torch.arange(tokens, device="cuda"), torch.zeros(tokens, dtype=torch.int32, device="cuda")
    freq, out, eager = D.rotary_frequency(32), torch.empty_like(q), torch.empty_like(q)
    side = torch.cuda.Stream()
    D.kv_append(a, k, v, slots, position, freq, q, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.kv_append(a, k, v, slots, position, freq, q, out)
    for turn in range(5):
        position.random_(0, 1 << 20)
        slots.copy_(torch.randperm(256, device="cuda")[:tokens])
        k.normal_()
        for c in (a, b):
            c.k.zero_(), c.v.zero_(), c.k_step.zero_(), c.v_step.zero_()
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        D.kv_append(b, k, v, slots, position, freq, q, eager, stream=side)
        side.synchronize()
        assert torch.equal(out, eager)
        for x, y in zip((a.k, a.v, a.k_step, a.v_step), (b.k, b.v, b.k_step, b.v_step)):
            assert torch.equal(x, y)


def test_no_tokens():
    import torch
    from paper_2507_12205_amd import device as D
    cache = D.kv_cache(1, 2, 16, 32, 8)
    x = torch.empty((0, 2, 32), dtype=torch.float16, device="cuda")
    D.kv_append(cache, x, x, torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), D.rotary_frequency(8), x)
    torch.cuda.synchronize()
    assert not cache.k.any()


@pytest.mark.parametrize("neighbours", [False, True])
def test_one_tensor_of_queries_keys_and_values(neighbours):
    """q, k and v as slices of one tensor, the queries rotated where they lie: nothing else of it changes."""
    import torch
    from paper_2507_12205_amd import device as D
    a, b = (D.kv_cache(9, 2, 16, 64, 16) for _ in range(2))
    both = values((50, 8, 64), 6, torch)
    before = both.clone()
    slots, position, freq = torch.arange(50, device="cuda"), torch.arange(7, 57, dtype=torch.int32, device="cuda"), D.rotary_frequency(32)
    want = D.kv_append(a, *(before[:, i:j].contiguous() for i, j in ((4, 6), (6, 8))), slots, position, freq, before[:, :4].contiguous(), None, neighbours)
    D.kv_append(b, both[:, 4:6], both[:, 6:], slots, position, freq, both[:, :4], None, neighbours)
    assert torch.equal(both[:, :4], want) and torch.equal(both[:, 4:], before[:, 4:]) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
