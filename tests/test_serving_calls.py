"""The Python calls around the products without a GPU: what they hand to the C ABI and what they refuse, on tensors of the CPU whose
addresses nothing looks at."""
import random

import pytest
import torch

from paper_2507_12205_amd import binding as B
from paper_2507_12205_amd import device as D


class Stream:
    cuda_stream = 0x55


@pytest.fixture
def calls(monkeypatch):
    """The descriptions and workspaces that reach the C ABI, in order."""
    seen = []
    monkeypatch.setattr(D.B, "ecspmv_attention", lambda cache, a, work, size, stream: seen.append((a, work, size, stream)))
    monkeypatch.setattr(D.B, "ecspmv_verify", lambda a, work, size, stream: seen.append((a, work, size, stream)))
    monkeypatch.setattr(D, "_stream_handle", lambda stream=None: 0 if stream is None else stream.cuda_stream)
    return seen


def cache(pages=8, heads=2, page=16, dim=64):
    """A cache of 16 bits as KvCache holds it, in host memory."""
    c = object.__new__(D.KvCache)
    c.bits, c.pages, c.heads, c.page_size, c.head_dim, c.device = 16, pages, heads, page, dim, -1
    c.k, c.v = (torch.zeros((pages, heads, page, dim), dtype=torch.float16) for _ in range(2))
    c.desc = B.KvCacheDesc(D._KV_CACHE, 16, pages, heads, page, dim, 0x100000, 0x200000, None, None)
    return c


def attention(c, table, q_heads=4, workspace=None, stream=None):
    batch = table.shape[0]
    q = torch.zeros((batch, q_heads, c.head_dim), dtype=torch.float16)
    return D.attention(c, q, torch.empty_like(q), torch.arange(batch + 1, dtype=torch.int32), torch.full((batch,), 3, dtype=torch.int32), table, 1,
                       workspace=workspace, stream=stream)


def test_rows_of_the_page_table_lie_apart(calls):
    """Rows that start less than their length apart (a table shared by expand(), overlapping rows) are refused: the C ABI has no such
    stride, and another in its place would have the later sequences' pages read from behind the table."""
    c, one = cache(), torch.arange(4, dtype=torch.int32)
    for table in (one[None].expand(3, -1), torch.arange(8, dtype=torch.int32).as_strided((3, 4), (2, 1))):
        with pytest.raises(AssertionError):
            attention(c, table)
    assert not calls
    wide = torch.arange(30, dtype=torch.int32).view(3, 10)
    for table, stride in ((wide, 10), (wide[:, :4], 10), (one[None], 4), (one[None].as_strided((1, 4), (0, 1)), 4), (wide[:1, :4], None),
                          (wide[:0], None), (wide[:, :1], 10), (wide[:, :0], None)):
        attention(c, table)
        a = calls.pop()[0]
        assert a.page_table == table.data_ptr() or table.numel() == 0
        assert a.table_stride >= a.max_pages == table.shape[1] and (stride is None or a.table_stride == stride)


@pytest.mark.parametrize("call", ["attention", "verify"])
def test_workspace_of_the_launch_s_stream(calls, monkeypatch, call):
    """A workspace that the call makes itself comes from the pool of the stream that the kernels run on: a block of another stream's pool may
    still be in use by that stream's kernels."""
    current, made = [None], []

    class On:
        def __init__(self, stream): self.stream = stream
        def __enter__(self): current.append(self.stream)
        def __exit__(self, *_): current.pop()
    monkeypatch.setattr(torch.cuda, "stream", On)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: (made.append(current[-1]), empty(*a, **k))[1])
    for stream in (None, Stream()):
        if call == "attention":
            c, table = cache(), torch.arange(4, dtype=torch.int32)[None]
            q, out = (torch.zeros((1, 4, 64), dtype=torch.float16) for _ in range(2))
            ints = [torch.tensor(v, dtype=torch.int32) for v in ([0, 1], [3])]
            D.attention(c, q, out, *ints, table, 1, stream=stream)
        else:
            p, q, x, u = torch.zeros(2, 4, 50), torch.zeros(2, 3, 50), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 4)
            monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
            D.verify(p, q, x, u, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), stream=stream)
        assert made == [stream] and calls.pop()[3] == (0x55 if stream else 0)
        made.clear()


def test_a_given_workspace_is_looked_at(calls, monkeypatch):
    """Its device and whether it is one piece; its size in bytes, whatever its type."""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: getattr(self, "place", 0))
    c, table = cache(), torch.arange(4, dtype=torch.int32)[None]
    c.device = 0
    p, q, x, u = torch.zeros(2, 4, 50), torch.zeros(2, 3, 50), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 4)
    tokens, accepted = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    elsewhere = torch.zeros(64, dtype=torch.uint8)
    elsewhere.place = -1
    for work in (elsewhere, torch.zeros(128, dtype=torch.uint8)[::2], torch.zeros(1, dtype=torch.uint8).expand(64)):
        with pytest.raises(AssertionError):
            attention(c, table, workspace=work)
        with pytest.raises(AssertionError):
            D.verify(p, q, x, u, tokens, accepted, workspace=work)
    assert not calls
    for work in (torch.zeros(64, dtype=torch.uint8), torch.zeros(8, dtype=torch.float64), torch.zeros((2, 8), dtype=torch.int32)):
        attention(c, table, workspace=work)
        D.verify(p, q, x, u, tokens, accepted, workspace=work)
        assert [k[1:3] for k in calls] == [(work.data_ptr(), 64)] * 2
        calls.clear()


@pytest.mark.parametrize("bits,heads,q_heads,dim", [(16, 32, 32, 128), (8, 8, 64, 128), (4, 2, 16, 96), (16, 1, 8, 256), (8, 1, 200, 64), (4, 40, 40, 64)])
@pytest.mark.parametrize("batch,max_new,max_kv", [(32, 1, 4096), (4, 8, 30000), (32, 2048, 4096), (5, 333, 3000), (1, 2048, 100000), (3, 40, 200)])
def test_a_workspace_for_all_smaller_calls(bits, heads, q_heads, dim, batch, max_new, max_kv):
    """Made once for the largest sizes, it holds for fewer sequences, tokens, new tokens of one and places too (which have more splits)."""
    c = cache(heads=heads, dim=dim)
    c.desc.bits, c.desc.k_step, c.desc.v_step = bits, 0x300000, 0x400000
    most = min(batch * max_new, (1 << 31) // q_heads - 1)
    have = D.attention_workspace(c, torch.empty((most, q_heads, dim), dtype=torch.float16, device="meta"), batch, max_new, max_kv).nbytes
    rng, need = random.Random(batch * max_new), 0
    sizes = [(b, n, kv) for b in range(1, batch + 1) for n in (1, (max_new + 1) // 2, max_new) for kv in (300, max_kv)]
    sizes += [(rng.randint(1, batch), rng.randint(1, max_new), rng.randint(1, max_kv)) for _ in range(2000)]
    for b, n, kv in sizes:
        tokens = rng.choice([b * n, rng.randint(n, b * n)])
        a = B.AttentionDesc(D._ATTENTION, q_heads, tokens, b, -(-min(kv, max_kv) // 16), n)
        need = max(need, B.ecspmv_attention_workspace(c.desc, a))
        assert need <= have, (b, n, kv, tokens)
    assert have <= 150 << 20                                 # and is not out of proportion


def test_products_with_an_epilogue_of_the_matrix_s_size(monkeypatch):
    """x, y and what the epilogue reads are looked at for their size and device: the kernel goes by the matrix."""
    import numpy as np
    mat = B.ecspmv_build_dense(np.eye(16, 128, dtype=np.float16), B.make_opts())
    seen = []
    monkeypatch.setattr(B.Matrix, "ecspmv_run_epilogue", lambda self, *a: seen.append(a))
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: getattr(self, "place", 0))
    monkeypatch.setattr(D, "_stream_handle", lambda stream=None: 0)

    def half(*shape, place=0):
        t = torch.zeros(shape, dtype=torch.float16)
        t.place = place
        return t
    right = dict(x=half(128, 4), y=half(16, 4), bias=half(16), gate=half(16, 4), residual=half(16, 4))
    D.run_epilogue(mat, **right)
    D.run_epilogue(mat, half(128), half(16))
    assert len(seen) == 2
    for wrong in (dict(x=half(127, 4)), dict(x=half(129, 4)), dict(y=half(15, 4), bias=None, gate=None, residual=None),
                  dict(y=half(17, 4), bias=half(17), gate=half(17, 4), residual=half(17, 4)), dict(x=half(128, 4, place=1)),
                  dict(bias=half(16, place=1)), dict(gate=half(16, 4, place=1)), dict(residual=half(16, 4, place=1))):
        with pytest.raises(AssertionError):
            D.run_epilogue(mat, **{**right, **wrong})
    assert len(seen) == 2
