"""PyTorch plumbing around the C ABI: device buffers and streams only, no arithmetic."""
from __future__ import annotations

from ctypes import sizeof

import numpy as np
import torch
from torch import _C

from . import binding as B


def _stream_handle(stream=None) -> int:
    """The HIP stream to launch on: the given one, or the current one of the current device (asked for as a plain handle:
    building torch's stream object takes 2.8 us, as long as the launch itself).  Only a call without a stream needs these two
    private functions of torch."""
    if stream is not None:
        return int(stream.cuda_stream)
    return _C._cuda_getCurrentRawStream(_C._cuda_getDevice())


def upload(mat: B.Matrix, device="cuda:0", stream=None) -> torch.Tensor:
    """Allocate the device image with PyTorch, copy the EC-CSR image into it, return the buffer."""
    nbytes = mat.ecspmv_device_bytes()
    buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
    assert buf.data_ptr() % 256 == 0
    mat.ecspmv_upload(buf.data_ptr(), nbytes, _stream_handle(stream), keepalive=buf)
    return buf


def run(mat: B.Matrix, x: torch.Tensor, y: torch.Tensor, stream=None) -> torch.Tensor:
    """y = W x on the given (or current) stream; x, y are CUDA tensors of length n, m: FP16, or FP32 for a matrix
    built from FP32 values."""
    want = torch.float32 if mat.value_bits == 32 else torch.float16
    assert x.dtype is want and y.dtype is want and x.is_cuda and y.is_cuda
    assert x.is_contiguous() and y.is_contiguous()
    mat.ecspmv_run(x.data_ptr(), y.data_ptr(), _C._cuda_getCurrentRawStream(_C._cuda_getDevice()) if stream is None else _stream_handle(stream))
    return y


def run_multi(mat: B.Matrix, X: torch.Tensor, Y: torch.Tensor, stream=None) -> torch.Tensor:
    """Y = W X for X of shape (n, nb), Y of shape (m, nb), row-major, nb in {1, 2, 4, 8}; FP16, or FP32 for a matrix
    built from FP32 values."""
    want = torch.float32 if mat.value_bits == 32 else torch.float16
    assert X.dtype is want and Y.dtype is want and X.is_cuda and Y.is_cuda
    assert X.dim() == 2 and Y.dim() == 2 and X.shape[1] == Y.shape[1] and X.is_contiguous() and Y.is_contiguous()
    mat.ecspmv_run_multi(X.data_ptr(), Y.data_ptr(), X.shape[1],
                         _C._cuda_getCurrentRawStream(_C._cuda_getDevice()) if stream is None else _stream_handle(stream))
    return Y


_EPILOGUE = sizeof(B.Epilogue)
_ACTIVATIONS = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}


def run_epilogue(mat: B.Matrix, x: torch.Tensor, y: torch.Tensor, bias: torch.Tensor = None, activation: str = "none",
                 gate: torch.Tensor = None, residual: torch.Tensor = None, stream=None) -> torch.Tensor:
    """y = activation(W x + bias) * gate + residual in one launch, each of the four left out where it is not given.  x (n,) and y (m,), or
    (n, nb) and (m, nb) with nb in {1, 2, 4, 8}; bias (m,); gate and residual shaped as y, which either may be itself; all FP16, or FP32 for
    a matrix built from FP32 values.  activation: "none", "relu", "gelu" (with the error function) or "silu"."""
    want = torch.float32 if mat.value_bits == 32 else torch.float16
    device, shape, e = x.get_device(), y.shape, B.Epilogue(_EPILOGUE, _ACTIVATIONS[activation])
    assert x.dtype is want and y.dtype is want and device >= 0 and y.get_device() == device and x.is_contiguous() and y.is_contiguous()
    assert x.dim() == y.dim() and x.shape[1:] == shape[1:] and len(shape) in (1, 2) and x.shape[0] == mat.n and shape[0] == mat.m
    if bias is not None:
        assert bias.dtype is want and bias.get_device() == device and bias.shape == shape[:1] and bias.is_contiguous()
        e.bias = bias.data_ptr()
    if gate is not None:
        assert gate.dtype is want and gate.get_device() == device and gate.shape == shape and gate.is_contiguous()
        e.gate = gate.data_ptr()
    if residual is not None:
        assert residual.dtype is want and residual.get_device() == device and residual.shape == shape and residual.is_contiguous()
        e.residual = residual.data_ptr()
    mat.ecspmv_run_epilogue(x.data_ptr(), y.data_ptr(), shape[1] if len(shape) == 2 else 1, e, _stream_handle(stream))
    return y


def csr_upload(csr: B.CsrMatrix, device="cuda:0", stream=None) -> torch.Tensor:
    nbytes = csr.ecspmv_csr_device_bytes()
    buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
    csr.ecspmv_csr_upload(buf.data_ptr(), nbytes, _stream_handle(stream), keepalive=buf)
    return buf


def csr_run(csr: B.CsrMatrix, x: torch.Tensor, y: torch.Tensor, stream=None) -> torch.Tensor:
    assert x.dtype == torch.float16 and y.dtype == torch.float16 and x.is_cuda and y.is_cuda
    csr.ecspmv_csr_run(x.data_ptr(), y.data_ptr(), _stream_handle(stream))
    return y


# ---- around the products ---------------------------------------------------------------------------------

_VIEW, _KV_CACHE, _ATTENTION, _VERIFY = (sizeof(t) for t in (B.View, B.KvCacheDesc, B.AttentionDesc, B.VerifyDesc))
_ROTARY, _KEEP, _VERIFY_TREE = (sizeof(t) for t in (B.RotaryDesc, B.KeepDesc, B.VerifyTreeDesc))


class KvCache:
    """A cache of keys and values in pages.  k, v: (pages, heads, page_size, head_dim) FP16 for 16 bits, int8 for 8;
    (pages, heads, page_size, head_dim / 2) uint8 for 4, the earlier code in the low half.  k_step, v_step: (pages, heads, page_size)
    FP32 for 8 bits, (pages, heads, page_size, 2) FP16, step and lowest value, for 4.  The tensors are the caller's and stay in place."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_step: torch.Tensor = None, v_step: torch.Tensor = None):
        self.bits = {torch.float16: 16, torch.int8: 8, torch.uint8: 4}[k.dtype]
        self.pages, self.heads, self.page_size, width = k.shape
        self.head_dim = 2 * width if self.bits == 4 else width
        assert v.dtype is k.dtype and v.shape == k.shape and k.is_cuda and v.device == k.device
        assert k.is_contiguous() and v.is_contiguous()
        if self.bits == 16:
            assert k_step is None and v_step is None
        else:
            want = (torch.float32, k.shape[:3]) if self.bits == 8 else (torch.float16, (*k.shape[:3], 2))
            for t in (k_step, v_step):
                assert t.dtype is want[0] and t.shape == want[1] and t.is_contiguous() and t.device == k.device
        self.k, self.v, self.k_step, self.v_step, self.device = k, v, k_step, v_step, k.get_device()
        self.desc = B.KvCacheDesc(_KV_CACHE, self.bits, self.pages, self.heads, self.page_size, self.head_dim, k.data_ptr(), v.data_ptr(),
                                  k_step.data_ptr() if k_step is not None else None, v_step.data_ptr() if v_step is not None else None)


def kv_cache(pages: int, heads: int, page_size: int, head_dim: int, bits: int = 16, device="cuda:0") -> KvCache:
    """An empty cache (all zeros)."""
    dtype, width = {16: (torch.float16, head_dim), 8: (torch.int8, head_dim), 4: (torch.uint8, head_dim // 2)}[bits]
    k, v = (torch.zeros((pages, heads, page_size, width), dtype=dtype, device=device) for _ in range(2))
    if bits == 16:
        return KvCache(k, v)
    dtype, shape = (torch.float32, (pages, heads, page_size)) if bits == 8 else (torch.float16, (pages, heads, page_size, 2))
    return KvCache(k, v, *(torch.zeros(shape, dtype=dtype, device=device) for _ in range(2)))


# These calls follow one another as fast as the host makes them, so devices are compared as plain numbers (-1: not on a GPU) and the
# structs are handed over as they are.

def _view(t: torch.Tensor) -> B.View:
    return B.View(t.data_ptr(), *t.stride())


def _workspace(nbytes: int, beside: torch.Tensor, stream) -> torch.Tensor:
    """Memory for one call, from the pool of the stream that it runs on: what is freed there is used again behind the call, and what is handed
    out there was freed before it.  (A block of the current stream's pool may still be in use by that stream's kernels.)"""
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=beside.device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=beside.device)


def _rows_of(cache: KvCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
    assert k.dtype is v.dtype is torch.float16 and k.get_device() == v.get_device() == slots.get_device() == cache.device
    assert k.shape == v.shape == (*slots.shape, cache.heads, cache.head_dim)
    assert slots.dtype is torch.int64 and slots.is_contiguous()


def kv_write(cache: KvCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, stream=None) -> None:
    """Keys and values of new tokens, (tokens, heads, head_dim) FP16 with any strides, into the places slots names: page * page_size +
    place in the page (int64, one per token; one outside the cache leaves its token out)."""
    _rows_of(cache, k, v, slots)
    B.ecspmv_kv_write(cache.desc, _view(k), _view(v), slots.data_ptr(), slots.shape[0], _stream_handle(stream))


def kv_read(cache: KvCache, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None):
    """The same places back into k and v (zeros for a place outside the cache)."""
    _rows_of(cache, k, v, slots)
    B.ecspmv_kv_read(cache.desc, slots.data_ptr(), slots.shape[0], _view(k), _view(v), _stream_handle(stream))
    return k, v


def kv_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, position: torch.Tensor, frequency: torch.Tensor,
              q: torch.Tensor = None, q_out: torch.Tensor = None, neighbours: bool = False, stream=None):
    """kv_write() of keys that are rotated by their tokens' positions, (tokens,) int32, on the way; queries q, (tokens, q_heads, head_dim) FP16 with
    any strides, are rotated into q_out (q itself if not given; not one that is expand()ed), which is returned.  frequency: (pairs,) FP64 radians a position (rotary_frequency());
    pair i of a head is its values i and i + pairs, or with `neighbours` values 2 i and 2 i + 1; the values beyond 2 * pairs stay as they are."""
    device, shape = cache.device, k.shape
    assert k.dtype is v.dtype is torch.float16 and slots.dtype is torch.int64 and position.dtype is torch.int32 and frequency.dtype is torch.float64
    assert device == k.get_device() == v.get_device() == slots.get_device() == position.get_device() == frequency.get_device()
    tokens, pairs = slots.numel(), frequency.numel()
    assert shape == v.shape == (tokens, cache.heads, cache.head_dim) and slots.dim() == position.dim() == frequency.dim() == 1
    assert position.numel() == tokens and slots.is_contiguous() and position.is_contiguous() and frequency.is_contiguous()
    if q is None:
        assert q_out is None
        r = B.RotaryDesc(_ROTARY, 2 * pairs, neighbours, 0, frequency.data_ptr(), position.data_ptr())
    else:
        if q_out is None:
            q_out = q
        q_tokens, q_heads, dim = q.shape
        assert q.dtype is q_out.dtype is torch.float16 and device == q.get_device() == q_out.get_device()
        assert q_tokens == tokens and dim == cache.head_dim and q_out.shape == q.shape
        r = B.RotaryDesc(_ROTARY, 2 * pairs, neighbours, q_heads, frequency.data_ptr(), position.data_ptr(), q.data_ptr(), *q.stride(),
                         q_out.data_ptr(), *q_out.stride())
    B.ecspmv_kv_append(cache.desc, B.View(k.data_ptr(), *k.stride()), B.View(v.data_ptr(), *v.stride()), slots.data_ptr(), tokens, r, _stream_handle(stream))
    return q_out


def rotary_frequency(pairs: int, base: float = 10000.0, device="cuda:0") -> torch.Tensor:
    """base ** (-i / pairs), for kv_append()."""
    return base ** (-torch.arange(pairs, dtype=torch.float64, device=device) / pairs)


class KvCaches:
    """The caches of a model's layers, alike but for their memory, which none shares with another, for kv_keep()."""

    def __init__(self, caches):
        self.caches = list(caches)
        assert self.caches and all((c.bits, c.pages, c.heads, c.page_size, c.head_dim, c.device) == self._shape() for c in self.caches)
        # rows of different caches move at the same time: no two of their tensors, which are contiguous, overlap
        tensors = [t for c in self.caches for t in ((c.k, c.v) if c.bits == 16 else (c.k, c.v, c.k_step, c.v_step))]
        spans = sorted((t.data_ptr(), t.data_ptr() + t.nbytes) for t in tensors)
        assert all(end <= start for (_, end), (start, _) in zip(spans, spans[1:]))
        self.device, self.descs = self.caches[0].device, B.cache_array([c.desc for c in self.caches])

    def _shape(self):
        c = self.caches[0]
        return c.bits, c.pages, c.heads, c.page_size, c.head_dim, c.device


def kv_keep(caches: KvCaches, first: torch.Tensor, path: torch.Tensor, accepted: torch.Tensor, page_table: torch.Tensor, stream=None) -> None:
    """The rows of accepted nodes to where they follow one another, in all caches: key first[b] + path[b, i] of sequence b becomes its key
    first[b] + i for i < accepted[b].  first: (batch,), the key of node 0; path: (batch, nodes) and accepted: (batch,) as verify_tree() leaves
    them; page_table as in attention(); all int32."""
    device, (batch, nodes), (sequences, pages), (row, node), (pages_row, place) = caches.device, path.shape, page_table.shape, path.stride(), page_table.stride()
    assert first.dtype is path.dtype is accepted.dtype is page_table.dtype is torch.int32
    assert device == first.get_device() == path.get_device() == accepted.get_device() == page_table.get_device()
    assert first.numel() == accepted.numel() == sequences == batch and first.dim() == accepted.dim() == 1
    assert first.is_contiguous() and accepted.is_contiguous()
    assert (nodes <= 1 or node == 1) and (batch <= 1 or row >= nodes) and (pages <= 1 or place == 1) and (batch <= 1 or pages_row >= pages)
    a = B.KeepDesc(_KEEP, batch, nodes, pages, row if batch > 1 else nodes, pages_row if batch > 1 else pages, first.data_ptr(), path.data_ptr(),
                   accepted.data_ptr(), page_table.data_ptr())
    B.ecspmv_kv_keep(caches.descs, a, _stream_handle(stream))


def attention_workspace(cache: KvCache, q: torch.Tensor, batch: int, max_new: int, max_kv: int) -> torch.Tensor:
    """A workspace for attention() and attention_tree() calls of up to these sizes: q's heads and no more tokens than it has (no more than batch * max_new if they
    are fewer), sequences, new tokens of one, places in their page tables."""
    a = B.AttentionDesc(_ATTENTION, q.shape[1], q.shape[0], batch, -(-max_kv // cache.page_size), max_new)
    return torch.empty(B.ecspmv_attention_workspace_most(cache.desc, a), dtype=torch.uint8, device=q.device)


def _attention_of(cache: KvCache, q: torch.Tensor, out: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor,
                  max_new: int, scale) -> B.AttentionDesc:
    device, (tokens, heads, dim), (batch, pages) = cache.device, q.shape, page_table.shape
    assert q.dtype is out.dtype is torch.float16 and q_start.dtype is kv_len.dtype is page_table.dtype is torch.int32
    assert device == q.get_device() == out.get_device() == q_start.get_device() == kv_len.get_device() == page_table.get_device()
    assert dim == cache.head_dim and out.shape == q.shape
    assert kv_len.numel() == batch and q_start.numel() == batch + 1 and kv_len.dim() == q_start.dim() == 1
    assert q_start.is_contiguous() and kv_len.is_contiguous()
    row, place = page_table.stride()
    assert (pages <= 1 or place == 1) and (batch <= 1 or row >= pages)          # no expand()ed rows
    return B.AttentionDesc(_ATTENTION, heads, tokens, batch, pages, max_new, dim ** -0.5 if scale is None else scale, row if batch > 1 else pages,
                           q_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), B.View(q.data_ptr(), *q.stride()),
                           B.View(out.data_ptr(), *out.stride()))


def attention(cache: KvCache, q: torch.Tensor, out: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor,
              max_new: int, scale: float = None, workspace: torch.Tensor = None, stream=None) -> torch.Tensor:
    """out = causal attention of the new tokens q, (tokens, q_heads, head_dim) FP16 with any strides, over the cache that holds their
    keys and values: sequence b has q[q_start[b]:q_start[b + 1]] and kv_len[b] keys in all, in the pages page_table[b] (all int32; rows of
    the table that do not overlap).
    max_new: the most new tokens of a sequence; scale: 1 / sqrt(head_dim) if not given."""
    a = _attention_of(cache, q, out, q_start, kv_len, page_table, max_new, scale)
    if workspace is None:
        workspace = _workspace(B.ecspmv_attention_workspace(cache.desc, a), q, stream)
    assert workspace.get_device() == cache.device and workspace.is_contiguous()
    B.ecspmv_attention(cache.desc, a, workspace.data_ptr(), workspace.nbytes, _stream_handle(stream))
    return out


def attention_tree(cache: KvCache, q: torch.Tensor, out: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor,
                   seen: torch.Tensor, max_new: int, scale: float = None, workspace: torch.Tensor = None, stream=None) -> torch.Tensor:
    """attention() of new tokens that are the nodes of a tree: each sees every key before the first new token of its sequence, and of the new tokens
    those whose bits are set in its row of seen, (tokens, words) int32 with 32 of them to a word, the first in the lowest bit (tree_seen()).
    words: no fewer than max_new / 32 (or, if there are fewer tokens than max_new, than those)."""
    a = _attention_of(cache, q, out, q_start, kv_len, page_table, max_new, scale)
    (tokens, words), (row, word) = seen.shape, seen.stride()
    assert seen.dtype is torch.int32 and seen.get_device() == cache.device and tokens == a.tokens and 32 * words >= min(max_new, tokens)
    assert (words <= 1 or word == 1) and (tokens <= 1 or row >= words)
    if workspace is None:
        workspace = _workspace(B.ecspmv_attention_tree_workspace(cache.desc, a), q, stream)
    assert workspace.get_device() == cache.device and workspace.is_contiguous()
    B.ecspmv_attention_tree(cache.desc, a, seen.data_ptr(), row if tokens > 1 else words, workspace.data_ptr(), workspace.nbytes,
                            _stream_handle(stream))
    return out


def tree_seen(parents, device="cuda:0") -> torch.Tensor:
    """The bits of attention_tree() of new tokens each of which sees itself and what its parent sees.  parents: a list for each sequence, of the number
    of each token's parent among the sequence's new tokens (less than its own; -1: none).  Worked out on the host."""
    count = sum(len(p) for p in parents)
    words = max([1] + [-(-len(p) // 32) for p in parents])
    seen, at = np.zeros((count, words), np.uint32), 0
    for of in parents:
        for i, p in enumerate(of):
            if not -1 <= p < i:
                raise ValueError(f"token {i} has the parent {p}")
            if p >= 0:
                seen[at + i] = seen[at + p]
            seen[at + i, i // 32] |= np.uint32(1 << i % 32)
        at += len(of)
    return torch.from_numpy(seen.view(np.int32)).to(device)


def verify_workspace(batch: int, vocab: int) -> int:
    """Bytes of a workspace for verify() calls of this size."""
    return B.ecspmv_verify_workspace(B.VerifyDesc(_VERIFY, batch, 0, vocab))


def verify(target: torch.Tensor, draft, drafted: torch.Tensor, uniform: torch.Tensor, tokens: torch.Tensor, accepted: torch.Tensor,
           count: torch.Tensor = None, workspace: torch.Tensor = None, stream=None):
    """Which drafted tokens stand, and the token after them.  target: (batch, drafts + 1, vocab) probabilities, draft: (batch, drafts,
    vocab) the drafts' own (None where a draft was certain), uniform: (batch, drafts + 1) random numbers in [0, 1), all FP32; drafted:
    (batch, drafts) int32, count: (batch,) int32, how many of them (None: all).  tokens: (batch, drafts + 1), accepted: (batch,) int32.
    workspace: of verify_workspace(), or allocated here."""
    batch, rows, vocab = target.shape
    drafts = rows - 1
    assert target.dtype is uniform.dtype is torch.float32 and drafted.dtype is tokens.dtype is accepted.dtype is torch.int32
    device = target.get_device()
    assert device >= 0 and device == uniform.get_device() == drafted.get_device() == tokens.get_device() == accepted.get_device()
    assert uniform.shape == tokens.shape == (batch, rows) and drafted.shape == (batch, drafts) and accepted.shape == (batch,)
    assert uniform.is_contiguous() and tokens.is_contiguous() and drafted.is_contiguous() and accepted.is_contiguous()
    assert target.numel() == 0 or vocab == 1 or target.stride(2) == 1
    a = B.VerifyDesc(_VERIFY, batch, drafts, vocab, target.data_ptr(), None, uniform.data_ptr(), target.stride(0), target.stride(1), 0, 0,
                     drafted.data_ptr() or None, None, tokens.data_ptr(), accepted.data_ptr())
    if draft is not None:
        assert draft.dtype is torch.float32 and draft.shape == (batch, drafts, vocab) and draft.get_device() == device
        assert draft.numel() <= 1 or vocab == 1 or draft.stride(2) == 1
        a.draft, a.draft_seq, a.draft_row = draft.data_ptr() or None, draft.stride(0), draft.stride(1)
    if count is not None:
        assert count.dtype is torch.int32 and count.shape == (batch,) and count.is_contiguous() and count.get_device() == device
        a.count = count.data_ptr()
    if workspace is None:
        workspace = _workspace(verify_workspace(batch, vocab), target, stream)
    assert workspace.get_device() == device and workspace.is_contiguous()
    B.ecspmv_verify(a, workspace.data_ptr(), workspace.nbytes, _stream_handle(stream))
    return tokens, accepted


def verify_tree_workspace(batch: int, nodes: int, vocab: int) -> int:
    """Bytes of a workspace for verify_tree() calls of this size."""
    return B.ecspmv_verify_tree_workspace(B.VerifyTreeDesc(_VERIFY_TREE, batch, nodes, vocab))


def verify_tree(target: torch.Tensor, drafted: torch.Tensor, parent: torch.Tensor, uniform: torch.Tensor, tokens: torch.Tensor, path: torch.Tensor,
                accepted: torch.Tensor, count: torch.Tensor = None, workspace: torch.Tensor = None, stream=None):
    """Which path of a tree of drafted tokens stands, and the token after it.  target: (batch, nodes + 1, vocab) probabilities, after the token before
    the tree and after each node, uniform: (batch, nodes + 1) random numbers in [0, 1), all FP32; drafted: (batch, nodes) and parent: (batch, nodes)
    int32, -1 for the token before the tree; count: (batch,) int32, how many nodes there are (None: all).  tokens: (batch, nodes + 1), path: (batch,
    nodes), accepted: (batch,) int32, which may be the memory of drafted, parent, count and uniform.  workspace: of verify_tree_workspace(), or allocated here."""
    device, (batch, rows, vocab), (seq, row, token) = target.get_device(), target.shape, target.stride()
    nodes = rows - 1
    assert target.dtype is uniform.dtype is torch.float32
    assert drafted.dtype is parent.dtype is tokens.dtype is path.dtype is accepted.dtype is torch.int32
    assert 0 <= device == uniform.get_device() == drafted.get_device() == parent.get_device()
    assert device == tokens.get_device() == path.get_device() == accepted.get_device()
    assert uniform.shape == tokens.shape == (batch, rows) and drafted.shape == parent.shape == path.shape == (batch, nodes) and accepted.shape == (batch,)
    assert uniform.is_contiguous() and tokens.is_contiguous() and drafted.is_contiguous() and parent.is_contiguous()
    assert path.is_contiguous() and accepted.is_contiguous() and (token == 1 or vocab == 1 or target.numel() == 0)
    a = B.VerifyTreeDesc(_VERIFY_TREE, batch, nodes, vocab, target.data_ptr(), uniform.data_ptr(), seq, row, drafted.data_ptr(), parent.data_ptr(), None,
                         tokens.data_ptr(), path.data_ptr(), accepted.data_ptr())
    if count is not None:
        assert count.dtype is torch.int32 and count.shape == (batch,) and count.is_contiguous() and count.get_device() == device
        a.count = count.data_ptr()
    if workspace is None:
        workspace = _workspace(B.ecspmv_verify_tree_workspace(a), target, stream)
    assert workspace.get_device() == device and workspace.is_contiguous()
    B.ecspmv_verify_tree(a, workspace.data_ptr(), workspace.nbytes, _stream_handle(stream))
    return tokens, path, accepted
