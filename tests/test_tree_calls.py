"""The Python calls of decoding with trees without a GPU: what they hand to the C ABI and what they refuse, on tensors of the CPU whose addresses
nothing looks at; the bits of a tree; and the registers of the kernels."""
import random
import re

import numpy as np
import pytest
import torch
import tree_reference as tree
from test_serving_calls import Stream, cache
from test_serving_registers import kernels

from paper_2507_12205_amd import binding as B
from paper_2507_12205_amd import device as D

I32, F32, F16, F64 = torch.int32, torch.float32, torch.float16, torch.float64


@pytest.fixture
def calls(monkeypatch):
    """What reaches the C ABI, in order."""
    seen = []
    for name in ("ecspmv_kv_append", "ecspmv_kv_keep", "ecspmv_attention_tree", "ecspmv_verify_tree"):
        monkeypatch.setattr(D.B, name, lambda *a, name=name: seen.append((name, a)))
    monkeypatch.setattr(D, "_stream_handle", lambda stream=None: 0 if stream is None else stream.cuda_stream)
    return seen


def elsewhere(t):
    """The same tensor, said to be on another device."""
    t = t.clone()
    t.place = 5
    return t


@pytest.fixture
def devices(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: getattr(self, "place", 0))


def refused(call, right, **wrongs):
    for name, values in wrongs.items():
        for value in values:
            with pytest.raises(AssertionError):
                call(**{**right, name: value})


def test_append(calls, devices):
    c = cache()
    c.device = 0
    half = lambda *s: torch.zeros(s, dtype=F16)                              # noqa: E731
    right = dict(cache=c, k=half(5, 2, 64), v=half(5, 2, 64), slots=torch.arange(5), position=torch.arange(5, dtype=I32),
                 frequency=torch.ones(20, dtype=F64), q=half(5, 6, 64), q_out=half(5, 6, 64), neighbours=True)
    assert D.kv_append(**right) is right["q_out"]
    (_, (desc, k, v, slots, tokens, r, stream)), = calls
    assert tokens == 5 and (r.rotary_dim, r.neighbours, r.q_heads) == (40, 1, 6) and r.frequency == right["frequency"].data_ptr()
    assert (r.q_token_stride, r.q_head_stride, r.q_dim_stride) == right["q"].stride() == (r.q_out_token_stride, r.q_out_head_stride, r.q_out_dim_stride)
    assert r.position == right["position"].data_ptr() and r.q == right["q"].data_ptr() and r.q_out == right["q_out"].data_ptr()
    calls.clear()
    assert D.kv_append(**{**right, "q_out": None, "neighbours": False}, stream=Stream()) is right["q"]
    (_, a), = calls
    assert a[5].q_out == right["q"].data_ptr() and a[5].neighbours == 0 and a[6] == 0x55
    calls.clear()
    assert D.kv_append(**{**right, "q": None, "q_out": None}) is None and calls.pop()[1][5].q_heads == 0
    wide = torch.zeros((5, 2), dtype=I32)
    refused(D.kv_append, right, position=[right["position"].long(), right["position"][:4], wide[:, 0], elsewhere(right["position"])],
            frequency=[right["frequency"].float(), torch.ones((40,), dtype=F64)[::2], elsewhere(right["frequency"])],
            q=[None, right["q"].float(), half(4, 6, 64), half(5, 6, 32), half(5, 5, 64), elsewhere(right["q"])], q_out=[half(5, 5, 64), half(5, 6, 64).float()],
            k=[half(4, 2, 64), half(5, 3, 64), half(5, 2, 64).float()], slots=[torch.arange(5, dtype=I32), torch.arange(4)])
    assert not calls


def test_keep(calls, devices):
    def at(shape=(8, 2, 16, 64)):
        c = cache(shape[0], shape[1], shape[2], shape[3])
        c.device = 0
        return c
    caches = D.KvCaches([at(), at(), at()])
    assert len(caches.descs) == 3 and caches.descs[2].contents.pages == 8
    for other in ((9, 2, 16, 64), (8, 1, 16, 64), (8, 2, 32, 64), (8, 2, 16, 48)):
        with pytest.raises(AssertionError):
            D.KvCaches([at(), at(other)])
    twice = at()
    for caches_of in ([], [twice, at(), twice]):
        with pytest.raises(AssertionError):
            D.KvCaches(caches_of)
    path, table = torch.zeros((2, 5), dtype=I32), torch.zeros((2, 4), dtype=I32)
    right = dict(caches=caches, first=torch.zeros(2, dtype=I32), path=path, accepted=torch.zeros(2, dtype=I32), page_table=table)
    D.kv_keep(**right)
    (_, (descs, a, stream)), = calls
    assert descs is caches.descs and (a.batch, a.nodes, a.max_pages, a.path_stride, a.table_stride) == (2, 5, 4, 5, 4)
    calls.clear()
    D.kv_keep(**{**right, "path": torch.zeros((2, 9), dtype=I32)[:, :5], "page_table": torch.zeros((2, 7), dtype=I32)[:, :4]}, stream=Stream())
    (_, (_, a, stream)), = calls
    assert (a.path_stride, a.table_stride, stream) == (9, 7, 0x55)
    calls.clear()
    refused(D.kv_keep, right, first=[torch.zeros(3, dtype=I32), torch.zeros(2), torch.zeros(4, dtype=I32)[::2], elsewhere(right["first"])],
            path=[path.long(), torch.zeros((5, 2), dtype=I32).t(), torch.zeros((1, 5), dtype=I32).expand(2, 5), elsewhere(path)],
            accepted=[torch.zeros(1, dtype=I32), elsewhere(right["accepted"])],
            page_table=[table[:1], torch.zeros((1, 4), dtype=I32).expand(2, 4), table.long(), elsewhere(table)])
    assert not calls


def test_caches_that_share_memory(devices):
    """Rows of different caches move at the same time: caches that overlap are refused, by whatever tensors; neighbours are not."""
    def at(k, v, k_step=None, v_step=None):
        c = cache(*k.shape)
        c.device, c.k, c.v = 0, k, v
        if k_step is not None:
            c.bits, c.k_step, c.v_step = 8, k_step, v_step
        return c
    k, v = (torch.zeros((24, 2, 16, 64), dtype=F16) for _ in range(2))
    D.KvCaches([at(k[:8], v[:8]), at(k[8:16], v[16:]), at(k[16:], v[8:16])])
    D.KvCaches([at(k[8 * i:8 * i + 8], k[8 * j:8 * j + 8]) for i, j in ((0, 2),)])
    for caches in ([at(k[:8], v[:8]), at(k[4:12], v[8:16])], [at(k[:8], v[:8]), at(k[8:16], v[7:15])], [at(k[:8], v[:8]), at(v[:8], k[8:16])],
                   [at(k[:8], k[:8])], [at(k[:8], v[:8]), at(k[8:16], v[8:16]), at(k[16:], k[15:23])]):
        with pytest.raises(AssertionError):
            D.KvCaches(caches)
    k, v = (torch.zeros((16, 2, 16, 64), dtype=torch.int8) for _ in range(2))
    ks, vs = (torch.zeros((16, 2, 16)) for _ in range(2))
    D.KvCaches([at(k[:8], v[:8], ks[:8], vs[:8]), at(k[8:], v[8:], ks[8:], vs[8:])])
    for steps in ((ks[:8], vs[8:]), (ks[8:], ks[:8]), (ks[7:15], vs[8:]), (ks[8:], vs[1:9])):
        with pytest.raises(AssertionError):
            D.KvCaches([at(k[:8], v[:8], ks[:8], vs[:8]), at(k[8:], v[8:], *steps)])


def test_attention(calls, devices, monkeypatch):
    monkeypatch.setattr(D.B, "ecspmv_attention_tree_workspace", lambda *a: 256)
    monkeypatch.setattr(D, "_workspace", lambda n, beside, stream: torch.zeros(n, dtype=torch.uint8))
    c = cache()
    c.device = 0
    q = torch.zeros((40, 4, 64), dtype=F16)
    right = dict(cache=c, q=q, out=torch.empty_like(q), q_start=torch.tensor([0, 40], dtype=I32), kv_len=torch.tensor([50], dtype=I32),
                 page_table=torch.arange(4, dtype=I32)[None], seen=torch.zeros((40, 2), dtype=I32), max_new=40)
    D.attention_tree(**right)
    (_, (_, a, seen, stride, work, size, stream)), = calls
    assert (seen, stride, size, a.max_new) == (right["seen"].data_ptr(), 2, 256, 40)
    calls.clear()
    D.attention_tree(**{**right, "seen": torch.zeros((40, 5), dtype=I32)[:, 1:3], "max_new": 1000}, stream=Stream())
    (_, a), = calls
    assert a[3] == 5 and a[6] == 0x55
    calls.clear()
    refused(D.attention_tree, right, seen=[right["seen"][:, :1], right["seen"][:39], right["seen"].long(), torch.zeros((1, 2), dtype=I32).expand(40, 2),
                                          torch.zeros((2, 40), dtype=I32).t(), elsewhere(right["seen"])],
            workspace=[elsewhere(torch.zeros(256, dtype=torch.uint8)), torch.zeros(512, dtype=torch.uint8)[::2]], out=[torch.zeros((40, 4, 32), dtype=F16)])
    assert not calls


def test_verify(calls, devices, monkeypatch):
    monkeypatch.setattr(D, "_workspace", lambda n, beside, stream: torch.zeros(n, dtype=torch.uint8))
    i32 = lambda *s: torch.zeros(s, dtype=I32)                                # noqa: E731
    right = dict(target=torch.zeros(2, 4, 50), drafted=i32(2, 3), parent=i32(2, 3), uniform=torch.zeros(2, 4), tokens=i32(2, 4), path=i32(2, 3),
                 accepted=i32(2), count=i32(2))
    assert D.verify_tree(**right) == (right["tokens"], right["path"], right["accepted"]) and D.verify_tree_workspace(3, 5, 2049) == 3 * (3 * 8 + 16 + 24)
    (_, (a, work, size, stream)), = calls
    assert (a.batch, a.nodes, a.vocab, a.target_seq, a.target_row, size) == (2, 3, 50, 200, 50, 2 * (8 + 16 + 16))
    assert a.parent == right["parent"].data_ptr() and a.path == right["path"].data_ptr() and a.count == right["count"].data_ptr()
    calls.clear()
    D.verify_tree(**{**right, "count": None, "target": torch.zeros(2, 5, 60)[:, :4, :50]}, stream=Stream())
    (_, (a, _, _, stream)), = calls
    assert (a.target_seq, a.target_row, a.count, stream) == (300, 60, None, 0x55)
    calls.clear()
    refused(D.verify_tree, right, target=[torch.zeros(2, 4, 50).double(), torch.zeros(2, 4, 100)[..., ::2], torch.zeros(2, 5, 50)],
            drafted=[i32(2, 4), i32(2, 3).long(), i32(3, 2).t(), elsewhere(i32(2, 3))], parent=[i32(2, 2), elsewhere(i32(2, 3)), i32(2, 6)[:, ::2]],
            uniform=[torch.zeros(2, 3), torch.zeros(2, 4).double()], tokens=[i32(2, 3), elsewhere(i32(2, 4))], path=[i32(2, 4), i32(2, 6)[:, ::2]],
            accepted=[i32(3), elsewhere(i32(2))], count=[i32(3), i32(2).long(), elsewhere(i32(2))], workspace=[elsewhere(torch.zeros(64, dtype=torch.uint8))])
    assert not calls


def test_the_bits_of_a_tree():
    rng = np.random.default_rng(3)
    for sizes in ([1], [64], [33, 1, 70], []):
        parents = [tree.parents(rng, n) for n in sizes]
        got, at = D.tree_seen(parents, device="cpu"), 0
        assert got.shape == (sum(sizes), max([1] + [-(-n // 32) for n in sizes])) and got.dtype is I32
        for p in parents:
            want = tree.pack(tree.tree_seen(p))
            assert np.array_equal(got[at:at + len(p), :want.shape[1]].numpy(), want) and not got[at:at + len(p), want.shape[1]:].any()
            at += len(p)
    for wrong in ([0], [-1, 1], [-1, -2], [-1, 5]):
        with pytest.raises(ValueError):
            D.tree_seen([wrong], device="cpu")


def test_frequencies():
    f = D.rotary_frequency(4, 10000.0, device="cpu")
    assert f.dtype is F64 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=F64))


def test_no_scratch_memory():
    found = {n: v for n, v in kernels().items() if any(x in n for x in ("kv_append", "kv_keep", "verify_tree", "attention_rows_kernel", "attention_chunk_kernel"))}
    assert len(found) > 40 and not {n: v for n, v in found.items() if v[1]}


def test_kernels_that_calls_reach():
    """Trees in heads of more than 128 have 64 rows to a workgroup: the library holds no kernel of 128 for them."""
    found = {tuple(map(int, m)) for n in kernels() for m in re.findall(r"attention_chunk_kernelILi(\d+)ELi(\d+)ELb1ELi(\d)EE", n)}
    assert found == {(bits, dim, on_keys) for bits in (16, 8, 4) for dim in range(32, 257, 32) for on_keys in (1, 2) if dim <= 128 or on_keys == 2}


@pytest.mark.parametrize("bits,heads,q_heads,dim", [(16, 32, 32, 128), (8, 8, 64, 128), (4, 2, 16, 96), (16, 1, 8, 256), (8, 1, 200, 64), (4, 40, 40, 64)])
@pytest.mark.parametrize("batch,max_new,max_kv", [(32, 1, 4096), (4, 8, 30000), (32, 64, 4096), (5, 333, 3000), (1, 257, 100000), (100, 40, 5000), (3, 40, 200)])
def test_a_workspace_for_all_smaller_calls(bits, heads, q_heads, dim, batch, max_new, max_kv):
    """Made once for the largest sizes, it holds for fewer sequences, tokens, new tokens of one and places too."""
    c, rng = cache(heads=heads, dim=dim), random.Random(batch * max_new)
    c.desc.bits, c.desc.k_step, c.desc.v_step = bits, 0x300000, 0x400000
    have = D.attention_workspace(c, torch.empty((batch * max_new, q_heads, dim), dtype=F16, device="meta"), batch, max_new, max_kv).nbytes
    sizes = [(b, n, kv) for b in range(1, batch + 1) for n in (1, (max_new + 1) // 2, max_new) for kv in (300, max_kv)]
    sizes += [(rng.randint(1, batch), rng.randint(1, max_new), rng.randint(1, max_kv)) for _ in range(2000)]
    for b, n, kv in sizes:
        tokens = rng.choice([b * n, rng.randint(n, b * n)])
        a = B.AttentionDesc(D._ATTENTION, q_heads, tokens, b, -(-min(kv, max_kv) // 16), n)
        assert B.ecspmv_attention_tree_workspace(c.desc, a) <= have, (b, n, kv, tokens)
