"""PyTorch plumbing around the C ABI: device buffers and streams only, no arithmetic."""
from __future__ import annotations

from ctypes import sizeof

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


def attention_workspace(cache: KvCache, q: torch.Tensor, batch: int, max_new: int, max_kv: int) -> torch.Tensor:
    """A workspace for attention() calls of up to these sizes: q's heads and no more tokens than it has (no more than batch * max_new if they
    are fewer), sequences, new tokens of one, places in their page tables."""
    a = B.AttentionDesc(_ATTENTION, q.shape[1], q.shape[0], batch, -(-max_kv // cache.page_size), max_new)
    return torch.empty(B.ecspmv_attention_workspace_most(cache.desc, a), dtype=torch.uint8, device=q.device)


def attention(cache: KvCache, q: torch.Tensor, out: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor,
              max_new: int, scale: float = None, workspace: torch.Tensor = None, stream=None) -> torch.Tensor:
    """out = causal attention of the new tokens q, (tokens, q_heads, head_dim) FP16 with any strides, over the cache that holds their
    keys and values: sequence b has q[q_start[b]:q_start[b + 1]] and kv_len[b] keys in all, in the pages page_table[b] (all int32; rows of
    the table that do not overlap).
    max_new: the most new tokens of a sequence; scale: 1 / sqrt(head_dim) if not given."""
    assert q.dtype is out.dtype is torch.float16 and q.shape == out.shape and q.shape[2] == cache.head_dim
    assert q.get_device() == out.get_device() == q_start.get_device() == kv_len.get_device() == page_table.get_device() == cache.device
    assert q_start.dtype is kv_len.dtype is page_table.dtype is torch.int32
    batch, pages = page_table.shape
    assert kv_len.shape == (batch,) and q_start.shape == (batch + 1,) and q_start.is_contiguous() and kv_len.is_contiguous()
    assert (pages <= 1 or page_table.stride(1) == 1) and (batch <= 1 or page_table.stride(0) >= pages)          # no expand()ed rows
    tokens, heads, _ = q.shape
    a = B.AttentionDesc(_ATTENTION, heads, tokens, batch, pages, max_new, cache.head_dim ** -0.5 if scale is None else scale,
                        page_table.stride(0) if batch > 1 else pages, q_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), _view(q), _view(out))
    if workspace is None:
        workspace = _workspace(B.ecspmv_attention_workspace(cache.desc, a), q, stream)
    assert workspace.get_device() == cache.device and workspace.is_contiguous()
    B.ecspmv_attention(cache.desc, a, workspace.data_ptr(), workspace.nbytes, _stream_handle(stream))
    return out


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
