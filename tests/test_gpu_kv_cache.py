"""The paged cache: what is written stands for the values that the definition gives, in place and nowhere else, and comes back."""
import numpy as np
import pytest
import serve_reference as ref

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 16, 16), (7, 3, 80, 16), (64, 12, 64, 32), (33, 2, 256, 64), (130, 8, 128, 256), (5, 1, 240, 1024)]   # tokens, heads, dim, page


def values(shape, seed, torch):
    x = np.random.default_rng(seed).normal(size=shape) * np.random.default_rng(seed + 1).choice([1e-3, 1.0, 30.0], size=(shape[0], shape[1], 1))
    return torch.from_numpy(x.astype(np.float16)).cuda()


def layout(x, kind, torch):
    """The same values in another layout: a column per token, heads first, rows that start off 16 bytes, a reversed order."""
    t, h, d = x.shape
    if kind == "columns":
        return x.permute(1, 2, 0).contiguous().permute(2, 0, 1)
    if kind == "heads":
        return x.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    if kind == "odd":
        wide = torch.empty((t, h, d + 3), dtype=x.dtype, device=x.device)
        wide[:, :, 1:d + 1] = x
        return wide[:, :, 1:d + 1]
    return x.clone()


def check(cache, x, code, step, slots, bits, back):
    """codes within what rounding a quotient in 32 bits can change: half a step and 2^-20 of the row's reach; steps to one last place"""
    page = cache.page_size
    got_code, got_step = code.cpu().numpy(), None if step is None else step.cpu().numpy()
    got = ref.decode(got_code, got_step, bits)
    x = x.cpu().numpy().astype(np.float64)
    for t, s in enumerate(slots):
        if not 0 <= s < cache.pages * page:
            assert not back[t].any()
            continue
        g = got[s // page, :, s % page]
        if bits == 16:
            assert np.array_equal(g, x[t]) and np.array_equal(back[t], x[t])
            continue
        _, want, low = ref.steps(x[t], bits)
        kept = got_step[s // page, :, s % page]
        kept_step = (kept if bits == 8 else kept[:, 0]).astype(np.float64)
        assert np.allclose(kept_step, want, rtol=2e-7 if bits == 8 else 1e-3, atol=0 if bits == 8 else 6e-8)
        if bits == 4:
            assert np.array_equal(kept[:, 1].astype(np.float64), low)
        # 4 bits: the step is rounded to 16 bits, so the last code may end 15 * 2^-11 steps from the largest value
        reach = np.abs(x[t]).max(-1, keepdims=True) + 1e-30
        slack = 0.5 * kept_step[:, None] * (1 if bits == 8 else 1 + 30 * 2 ** -11) + 2 ** -20 * reach + (0 if bits == 8 else 15 * 6e-8)
        assert (np.abs(g - x[t]) <= slack).all()
        assert np.array_equal(back[t], (got.astype(np.float32)[s // page, :, s % page]).astype(np.float16)) or \
            (np.abs(back[t].astype(np.float64) - g) <= 2 ** -11 * np.abs(g) + 6e-8).all()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("kind", ["plain", "columns", "heads", "odd"])
@pytest.mark.parametrize("shape", SHAPES)
def test_write_and_read(shape, kind, bits):
    import torch
    from paper_2507_12205_amd import device as D
    tokens, heads, dim, page = shape
    pages = 2 * (-(-tokens // page)) + 1
    cache = D.kv_cache(pages, heads, page, dim, bits)
    for t in (cache.k, cache.v, cache.k_step, cache.v_step):
        if t is not None:
            t.fill_(3)                                       # what is not written stays as it was
    k, v = values((tokens, heads, dim), 1, torch), values((tokens, heads, dim), 5, torch)
    k[0, 0] = 0                                              # a row of zeros, one of equal values
    v[0, 0] = 0.75
    slots = np.random.default_rng(3).permutation(pages * page)[:tokens].astype(np.int64)
    if tokens > 6:
        slots[2], slots[5] = -1, pages * page
    before = [None if t is None else t.clone() for t in (cache.k, cache.v, cache.k_step, cache.v_step)]
    sd = torch.from_numpy(slots).cuda()
    D.kv_write(cache, layout(k, kind, torch), layout(v, kind, torch), sd)
    kb, vb = (layout(torch.full_like(k, float("nan")), kind, torch) for _ in range(2))
    D.kv_read(cache, sd, kb, vb)
    torch.cuda.synchronize()
    check(cache, k, cache.k, cache.k_step, slots, bits, kb.cpu().numpy())
    check(cache, v, cache.v, cache.v_step, slots, bits, vb.cpu().numpy())
    used = slots[(slots >= 0) & (slots < pages * page)]
    free = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    free[torch.from_numpy(used).cuda()] = False
    free = free.view(pages, page)
    for now, was in zip((cache.k, cache.v, cache.k_step, cache.v_step), before):
        if now is not None:
            assert torch.equal(now.transpose(1, 2)[free], was.transpose(1, 2)[free])


@pytest.mark.parametrize("bits", [8, 4])
def test_values_that_are_not_finite(bits):
    """NaN counts as 0, infinities as the largest FP16 value: every code stands for a finite value."""
    import torch
    from paper_2507_12205_amd import device as D
    cache = D.kv_cache(1, 1, 16, 32, bits)
    x = torch.randn(4, 1, 32, dtype=torch.float16, device="cuda")
    x[0, 0, 3], x[1, 0, 4], x[2, 0, 5], x[3, 0] = float("nan"), float("inf"), float("-inf"), float("nan")
    slots = torch.arange(4, device="cuda")
    D.kv_write(cache, x, x, slots)
    back, other = torch.empty_like(x), torch.empty_like(x)
    D.kv_read(cache, slots, back, other)
    assert torch.isfinite(back).all() and torch.equal(back, other)
    assert not back[3].any() and back[1, 0, 4] > 65000 and back[2, 0, 5] < -65000
    want = torch.nan_to_num(x[0].float(), 0.0)
    assert (back[0].float() - want).abs().max() <= (want.max() - want.min()) / (15 if bits == 4 else 127) * 0.6


def test_no_tokens():
    import torch
    from paper_2507_12205_amd import device as D
    cache = D.kv_cache(1, 2, 16, 32, 8)
    x = torch.empty((0, 2, 32), dtype=torch.float16, device="cuda")
    D.kv_write(cache, x, x, torch.empty(0, dtype=torch.int64, device="cuda"))
    D.kv_read(cache, torch.empty(0, dtype=torch.int64, device="cuda"), x, x)
    torch.cuda.synchronize()
    assert not cache.k.any()
