"""Products with bias, activation, gate and residual against 64 bits, and against the plain product where there is nothing to add.

The bound: the product's own band of FP32 sums (2^-17 of sum |w x|, as for products with FP32 values), carried through the activation (whose
slope stays under 1.13) and the gate, what the epilogue itself computes in FP32 (2^-20 of its terms), and the rounding of y."""
import math

import numpy as np
import pytest
from workloads import generators as gen

pytestmark = pytest.mark.gpu


def act(t, name):
    if name == "relu":
        return np.maximum(t, 0)
    if name == "silu":
        return t / (1 + np.exp(-t))
    if name == "gelu":
        return 0.5 * t * np.array([math.erfc(-v / math.sqrt(2)) for v in t.ravel()]).reshape(t.shape)
    return t


def matrix(m, n, density, fp32, seed, dense_rows=0):
    rng = np.random.default_rng(seed)
    W = np.where(rng.random((m, n)) < density, rng.normal(size=(m, n)) * 0.1, 0)
    if dense_rows:                                           # rows that share columns: block sets
        cols = np.sort(rng.permutation(n)[:max(64, n // 3)])
        for r in range(0, m - dense_rows, 2 * dense_rows):
            W[r:r + dense_rows, cols] = rng.normal(size=(dense_rows, len(cols))) * 0.1
    return W.astype(np.float32 if fp32 else np.float16)


def check(W, A, nb, fp32, name, bias, gate, residual, seed, inplace=""):
    import torch
    from paper_2507_12205_amd import device as D
    dt, td = (np.float32, torch.float32) if fp32 else (np.float16, torch.float16)
    m, n = W.shape
    rng = np.random.default_rng(seed)
    shape = (lambda r: (r,)) if nb == 1 else (lambda r: (r, nb))
    x, b, g, r = (rng.normal(size=s).astype(dt) for s in (shape(n), (m,), shape(m), shape(m)))
    put = lambda v: torch.from_numpy(v).cuda()               # noqa: E731
    y = torch.full(shape(m), float("nan"), dtype=td, device="cuda")
    gd, rd = put(g) if gate else None, put(r) if residual else None
    if inplace == "residual":
        y = rd
    elif inplace == "gate":
        y = gd
    D.run_epilogue(A, put(x), y, put(b) if bias else None, name, gd, rd)
    got = y.cpu().numpy().astype(np.float64)
    W64, x64 = W.astype(np.float64), x.astype(np.float64)
    t, size = W64 @ x64, np.abs(W64) @ np.abs(x64)
    wide = (lambda v: v) if nb == 1 else (lambda v: v[:, None])
    if bias:
        t = t + wide(b.astype(np.float64))
        size = size + wide(np.abs(b.astype(np.float64)))
    a = act(t, name)
    want = a * g if gate else a
    bound = 1.2 * 2 ** -17 * size * (np.abs(g.astype(np.float64)) if gate else 1.0) + 2 ** -20 * np.abs(want)
    if residual:
        want = want + r
        bound = bound + 2 ** -20 * np.abs(r.astype(np.float64))
    bound = bound + (2 ** -24 if fp32 else 2 ** -11) * np.abs(want) + (1e-30 if fp32 else 2 ** -24)
    worst = np.max(np.abs(got - want) / bound)
    assert worst <= 1.0, worst
    return y


SHAPES = [(1, 1, 1.0, 0, {}), (37, 65, 0.5, 0, {}), (300, 1000, 0.3, 0, {}), (520, 768, 0.4, 4, {}), (256, 700, 0.5, 8, dict(max_granularity=8)),
          (2000, 3000, 0.2, 2, {}), (100, 1000, 0.9, 0, dict(num_panels=1))]


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("nb", [1, 2, 4, 8])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_64_bits(shape, nb, fp32):
    from paper_2507_12205_amd import binding as B, device as D
    m, n, density, dense, opts = SHAPES[shape]
    if fp32:
        opts = {k: v for k, v in opts.items() if k != "max_granularity"}
    W = matrix(m, n, density, fp32, shape, dense)
    for bits in (4, 8):
        A = (B.ecspmv_build_dense_f32 if fp32 else B.ecspmv_build_dense)(W, B.make_opts(delta_bits=bits, **opts))
        D.upload(A)
        for k, (name, bias, gate, residual, inplace) in enumerate([
                ("none", True, False, True, "residual"), ("silu", False, True, False, "gate"), ("gelu", True, True, True, ""),
                ("relu", True, False, False, ""), ("none", False, False, True, ""), ("none", False, True, False, "")]):
            check(W, A, nb, fp32, name, bias, gate, residual, 10 * shape + k, inplace)


@pytest.mark.parametrize("opts,fp32", [(dict(delta_bits=16), False), (dict(max_granularity=16, flags=4), False), (dict(max_granularity=16, delta_bits=16, flags=4), False),
                                       (dict(max_granularity=16, flags=4), True)])
def test_formats_for_one_vector_only(opts, fp32):
    from paper_2507_12205_amd import binding as B, device as D
    W = matrix(400, 900, 0.3, fp32, 3, dense_rows=16)
    A = (B.ecspmv_build_dense_f32 if fp32 else B.ecspmv_build_dense)(W, B.make_opts(**opts))
    D.upload(A)
    check(W, A, 1, fp32, "gelu", True, True, True, 5)


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("nb", [1, 2, 4, 8])
def test_nothing_to_add_gives_the_products_bits(nb, fp32):
    """Without an epilogue, and with one that changes nothing in FP32 (a bias of zeros), y has the bits of the plain product."""
    import torch
    from paper_2507_12205_amd import binding as B, device as D
    for n, density in ((700, 0.4), (9000, 0.2)):             # (the wide one: rows of x come first, several workgroups a panel)
        W = matrix(300, n, density, fp32, n)
        A = (B.ecspmv_build_dense_f32 if fp32 else B.ecspmv_build_dense)(W)
        D.upload(A)
        td = torch.float32 if fp32 else torch.float16
        x = torch.randn((n, nb) if nb > 1 else (n,), device="cuda").to(td)
        y, z = (torch.empty((300, nb) if nb > 1 else (300,), dtype=td, device="cuda") for _ in range(2))
        D.run_multi(A, x, y) if nb > 1 else D.run(A, x, y)
        D.run_epilogue(A, x, z)
        assert torch.equal(y, z)
        D.run_epilogue(A, x, z, bias=torch.zeros(300, dtype=td, device="cuda"))
        assert torch.equal(y, z)


def test_rows_in_another_order_and_an_unaligned_x():
    import torch
    from paper_2507_12205_amd import binding as B, device as D
    W, x = gen.small_random(130, 500, 0.4, 7)
    A = B.ecspmv_build_dense(W, B.make_opts(flags=B.FLAG_CLUSTER_ROWS))
    D.upload(A)
    check(W, A, 1, False, "silu", True, True, True, 1)
    buf = torch.zeros(501, dtype=torch.float16, device="cuda")
    buf[1:] = torch.from_numpy(x).cuda()
    y, z, r = (torch.randn(130, device="cuda").half() for _ in range(3))
    D.run_epilogue(A, buf[1:], y, residual=r)
    D.run_epilogue(A, buf[1:].clone(), z, residual=r)
    assert torch.equal(y, z)


def test_special_values():
    """NaN passes relu; large negative values are 0 under silu and gelu; an infinite residual stays one."""
    import torch
    from paper_2507_12205_amd import binding as B, device as D
    A = B.ecspmv_build_dense_f32(np.eye(64, dtype=np.float32))
    D.upload(A)
    x = torch.zeros(64, device="cuda")
    x[1], x[2] = -200.0, 200.0
    y = torch.empty(64, device="cuda")
    bias = torch.zeros(64, device="cuda")
    bias[0] = float("nan")
    assert torch.isnan(D.run_epilogue(A, x, y, bias, "relu")[0]) and y[1] == 0 and y[2] == 200
    for name in ("silu", "gelu"):
        D.run_epilogue(A, x, y, None, name)
        assert y[1] == 0 and y[2] == 200
    res = torch.full((64,), float("inf"), device="cuda")
    assert torch.isinf(D.run_epilogue(A, x, y, None, "none", None, res)).all()


def test_in_a_graph_and_on_another_stream():
    import torch
    from paper_2507_12205_amd import binding as B, device as D
    W = matrix(200, 600, 0.3, False, 2)
    A = B.ecspmv_build_dense(W)
    D.upload(A)
    x, y, r, b = torch.randn(600, 4, device="cuda").half(), torch.empty(200, 4, device="cuda").half(), torch.randn(200, 4, device="cuda").half(), \
        torch.randn(200, device="cuda").half()
    side = torch.cuda.Stream()
    D.run_epilogue(A, x, y, b, "gelu", None, r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.run_epilogue(A, x, y, b, "gelu", None, r)
    for _ in range(3):
        x.normal_()
        r.normal_()
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        z = torch.empty_like(y)
        D.run_epilogue(A, x, z, b, "gelu", None, r, stream=side)
        side.synchronize()
        assert torch.equal(y, z) and torch.isfinite(y).all()
