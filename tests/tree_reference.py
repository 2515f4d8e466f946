"""The operators of decoding with trees of drafted tokens in 64 bits on the CPU, from their definitions, and random trees."""
import numpy as np
import serve_reference as ref


def parents(rng, nodes):
    """A random tree: each node's parent among those before it, -1 for the token before the tree."""
    return [int(rng.integers(-1, i)) if rng.random() < 0.5 else i - 1 for i in range(nodes)]


def pack(seen):
    """(tokens, new tokens) truth values as (tokens, words) int32."""
    tokens, count = seen.shape
    words = np.zeros((tokens, max(1, -(-count // 32))), np.uint32)
    for i in range(count):
        words[:, i // 32] |= seen[:, i].astype(np.uint32) << np.uint32(i % 32)
    return words.view(np.int32)


def tree_seen(parent):
    """(tokens, tokens): whether a token sees another, itself and what its parent sees."""
    seen = np.zeros((len(parent), len(parent)), bool)
    for i, p in enumerate(parent):
        if p >= 0:
            seen[i] = seen[p]
        seen[i, i] = True
    return seen


def rotate(x, position, frequency, neighbours):
    """(tokens, heads, dim) with the pairs as complex numbers, times exp(i position * frequency)."""
    x = np.asarray(x, np.float64).copy()
    pairs = len(frequency)
    turn = np.exp(1j * (np.asarray(position, np.float64)[:, None] * frequency))[:, None]
    first, second = (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if neighbours else (x[..., :pairs], x[..., pairs:2 * pairs])
    with np.errstate(invalid="ignore"):
        z = (first + 1j * second) * turn
    first[...], second[...] = z.real, z.imag
    return x


def attention(q, k, v, q_start, kv_len, table, seen, scale):
    """Result and the sum of p |v| of every value; seen: a (new tokens, new tokens) array of truth values for each sequence."""
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    group = q.shape[1] // k.shape[1]
    with np.errstate(invalid="ignore", over="ignore"):
        for b, n in enumerate(kv_len):
            kk, vv = (ref.gather(c, table[b], n) for c in (k, v))
            new = q_start[b + 1] - q_start[b]
            node = np.arange(n) - (n - new)                   # which new token a key is
            for t in range(new):
                see = np.array([i < 0 or bool(seen[b][t, i]) for i in node], bool)
                if not see.any():
                    continue
                for h in range(q.shape[1]):
                    a = scale * (kk[h // group, see] @ q[q_start[b] + t, h])
                    p = np.exp(a - a.max())
                    p /= p.sum()
                    out[q_start[b] + t, h] = p @ vv[h // group, see]
                    size[q_start[b] + t, h] = p @ np.abs(vv[h // group, see])
    return out, size


def verify(target, drafted, parent, uniform, count=None):
    batch, nodes = drafted.shape
    tokens, path = np.full((batch, nodes + 1), -1, np.int32), np.full((batch, nodes), -1, np.int32)
    accepted = np.zeros(batch, np.int32)
    for b in range(batch):
        k = nodes if count is None else min(max(int(count[b]), 0), nodes)
        at, n, go_on = -1, 0, True
        while go_on:
            p = np.maximum(np.nan_to_num(target[b, at + 1].astype(np.float64), posinf=np.inf), 0)
            left, gone, go_on = 1.0, set(), False
            for i in range(k):
                if parent[b, i] != at or parent[b, i] >= i:
                    continue
                x = int(drafted[b, i])
                if x in gone:
                    continue
                inside = 0 <= x < target.shape[2]
                if inside and float(uniform[b, i]) * left < p[x]:
                    path[b, n], tokens[b, n] = i, x
                    at, n, go_on = i, n + 1, True
                    break
                if inside:
                    left -= p[x]
                    gone.add(x)
        accepted[b] = n
        w = p.copy()
        w[list(gone)] = 0
        if not w.sum() > 0:
            w = p
        if w.sum() > 0:
            hit = np.nonzero(np.cumsum(w) > float(uniform[b, nodes]) * w.sum())[0]
            tokens[b, n] = hit[0] if len(hit) else np.nonzero(w)[0][-1]
    return tokens, path, accepted


def keep(tensors, first, path, accepted, table, page):
    """Moves rows in place, one after the other, in (pages, heads, page, ...) arrays."""
    pages = tensors[0].shape[0]
    for b in range(len(first)):
        for i in range(min(max(int(accepted[b]), 0), path.shape[1])):
            at, to = int(first[b]) + int(path[b, i]), int(first[b]) + i
            if path[b, i] <= i or first[b] < 0 or at >= table.shape[1] * page:
                continue
            pa, pt = int(table[b, at // page]), int(table[b, to // page])
            if 0 <= pa < pages and 0 <= pt < pages:
                for t in tensors:
                    t[pt, :, to % page] = t[pa, :, at % page]
