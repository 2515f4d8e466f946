"""The cache in 8 and 4 bits at the ends of FP16's range: every code stands for a value that FP16 holds."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ENDS = [(-65504.0, 65504.0), (-30000.0, 65504.0), (-65504.0, 30000.0), (-2.0, 65504.0), (0.0, 65504.0), (65472.0, 65504.0), (-65504.0, -65472.0),
        (-np.inf, np.inf), (-30000.0, np.inf), (-np.inf, 1.0), (-61000.0, 65000.0), (-6e-8, 6e-8), (60000.0, 65504.0)]


@pytest.mark.parametrize("bits", [8, 4])
def test_rows_that_reach_the_ends(bits):
    """Read back: finite, and half a step from what was written.  The step is that of the definition, or in 4 bits its neighbours in FP16
    (2^-10 of it), which the last code meets 15 times; FP16 rounds the result (2^-11 of it, 2^-25 below the normal range)."""
    import torch
    from paper_2507_12205_amd import device as D
    rng = np.random.default_rng(2)
    x = np.stack([np.clip(rng.uniform(max(a, -65504), min(b, 65504), 32), -65504, 65504) for a, b in ENDS]).astype(np.float16)
    for row, (a, b) in zip(x, ENDS):
        row[[3, 17]] = a, b
    cache = D.kv_cache(1, 1, 16, 32, bits)
    k = torch.from_numpy(x)[:, None].cuda()
    slots = torch.arange(len(ENDS), device="cuda")
    D.kv_write(cache, k, -k, slots)
    back, other = torch.empty_like(k), torch.empty_like(k)
    D.kv_read(cache, slots, back, other)
    for got, want in ((back, x), (other, -x)):
        got, want = got[:, 0].cpu().numpy().astype(np.float64), np.clip(want.astype(np.float64), -65504, 65504)
        assert np.isfinite(got).all()
        reach = np.abs(want).max(1) / 127 if bits == 8 else (want.max(1) - want.min(1)) / 15
        bound = reach * (0.5 + (0 if bits == 8 else 15 * 2 ** -10)) + 16 * 2 ** -24 + 2 ** -11 * np.abs(got).max(1)
        assert (np.abs(got - want).max(1) <= bound).all()


@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("bits", [8, 4])
def test_attention_over_them(bits, new):
    """One key repeated: the result is its value."""
    import torch
    from paper_2507_12205_amd import device as D
    for a, b in ENDS[:3]:
        row = torch.linspace(a, b, 64, device="cuda").half()
        cache = D.kv_cache(8, 1, 16, 64, bits)
        k = row.expand(new, 1, 64)
        D.kv_write(cache, torch.zeros_like(k), k, torch.arange(new, device="cuda"))
        back, other = torch.empty((new, 1, 64), dtype=torch.float16, device="cuda"), torch.empty((new, 1, 64), dtype=torch.float16, device="cuda")
        D.kv_read(cache, torch.arange(new, device="cuda"), other, back)
        out = torch.empty_like(back)
        ints = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, new], [new], [list(range(8))])]
        D.attention(cache, torch.ones_like(out), out, *ints, new)
        assert torch.isfinite(out).all()
        # FP16 of what was read back and of the result, weights as FP16 in one or two parts
        assert ((out - back).double().abs() <= 2 ** -9 * back.double().abs().max()).all()
