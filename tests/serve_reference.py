"""The operators around the products in 64 bits on the CPU, from their definitions: the cache, attention over it, the check of drafts."""
import numpy as np


def steps(x, bits):
    """(codes, step, low) of rows of values; the steps as they are kept (FP32 for 8 bits, FP16 for 4)."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), 0.0, np.clip(x, -65504.0, 65504.0))
    if bits == 8:
        step = (np.abs(x).max(-1).astype(np.float32) / np.float32(127)).astype(np.float64)
        safe = np.where(step > 0, step, 1.0)
        return np.where(step[..., None] > 0, np.rint(x / safe[..., None]), 0.0), step, np.zeros_like(step)
    low = x.min(-1)
    step = (((x.max(-1) - low).astype(np.float32) / np.float32(15)).astype(np.float16)).astype(np.float64)
    safe = np.where(step > 0, step, 1.0)
    return np.where(step[..., None] > 0, np.clip(np.rint((x - low[..., None]) / safe[..., None]), 0, 15), 0.0), step, low


def decode(codes, step_bits, bits):
    """Values of a cache's tensors (numpy, as they lie in memory)."""
    if bits == 16:
        return codes.astype(np.float64)
    if bits == 8:
        return codes.astype(np.float64) * step_bits.astype(np.float64)[..., None]
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1).astype(np.float64)
    return step_bits[..., 1:2].astype(np.float64) + step_bits[..., 0:1].astype(np.float64) * c


def gather(cache, table, length):
    """(heads, length, dim) of a sequence from the (pages, heads, page_size, dim) values of a cache."""
    _, heads, page, dim = cache.shape
    pages = cache[table[:-(-length // page)]]
    return pages.transpose(1, 0, 2, 3).reshape(heads, -1, dim)[:, :length]


def attention(q, k, v, q_start, kv_len, table, scale):
    """Result and, for the bound of its error, the sum of p |v| of every value."""
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    group = q.shape[1] // k.shape[1]
    with np.errstate(invalid="ignore", over="ignore"):
        for b, n in enumerate(kv_len):
            kk, vv = (gather(c, table[b], n) for c in (k, v))
            new = q_start[b + 1] - q_start[b]
            for t in range(new):
                seen = n - new + t + 1
                if seen <= 0:
                    continue
                for h in range(q.shape[1]):
                    a = scale * (kk[h // group, :seen] @ q[q_start[b] + t, h])
                    p = np.exp(a - a.max())
                    p /= p.sum()
                    out[q_start[b] + t, h] = p @ vv[h // group, :seen]
                    size[q_start[b] + t, h] = p @ np.abs(vv[h // group, :seen])
    return out, size


def verify(target, draft, drafted, uniform, count=None):
    batch, drafts = drafted.shape
    tokens, accepted = np.full((batch, drafts + 1), -1, np.int32), np.zeros(batch, np.int32)
    for b in range(batch):
        k = drafts if count is None else min(max(int(count[b]), 0), drafts)
        n = 0
        while n < k:
            x = int(drafted[b, n])
            if not 0 <= x < target.shape[2]:
                break
            q = np.float32(1) if draft is None else draft[b, n, x]
            if not np.float32(uniform[b, n]) * q < target[b, n, x]:
                break
            n += 1
        p = np.maximum(np.nan_to_num(target[b, n].astype(np.float64)), 0)
        w = p
        if n < k:
            if draft is None:
                w = p.copy()
                if 0 <= int(drafted[b, n]) < len(w):
                    w[int(drafted[b, n])] = 0
            else:
                w = np.maximum(p - draft[b, n].astype(np.float64), 0)
            if not w.sum() > 0:
                w = p
        accepted[b] = n
        tokens[b, :n] = drafted[b, :n]
        if w.sum() > 0:
            hit = np.nonzero(np.cumsum(w) > float(uniform[b, drafts]) * w.sum())[0]
            tokens[b, n] = hit[0] if len(hit) else np.nonzero(w)[0][-1]
    return tokens, accepted
