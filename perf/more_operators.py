"""The operators of decoding with a tree of drafted tokens, as timed cases: new keys rotated by their positions into the paged cache, the
attention of the tree's nodes over it, the check of the tree, and the accepted path's rows kept in the caches of all layers.

With `own` false they are computed in plain torch operations; with `own` true by the calls a serving program makes of this library.

A case is a dict:
  kind "append"  queries and keys of `tokens` new tokens rotated by their positions (from `past` on), keys and values into their places
       tokens, q_heads, heads (of keys and values), dim, rotary (values of a head that are rotated), neighbours (pairs are neighbouring
       values, not halves), page (tokens), bits (16, 8 or 4 for a cached value), past, tree (positions are depths in a tree), columns
  kind "tree"    attention of the waiting token and the drafted nodes of `batch` sequences, each seeing its own path and what came before
       batch, new (most new tokens of a sequence), past (most tokens before them), ragged (lengths from a tenth of that up),
       heads, kv_heads, dim, page, bits, columns (activations as the products leave them: one column per token)
  kind "check"   a tree of `nodes` drafted tokens of `batch` sequences against the target's probabilities over `vocab` tokens
       batch, nodes, vocab, ragged (fewer nodes in some sequences), greedy (the target's likeliest token is certain)
  kind "keep"    the rows of `kept` accepted of `nodes` drafted nodes moved behind the text, in the caches of `layers` layers
       layers, batch, nodes, kept, past, heads, dim, page, bits
"""
import math
import random

import numpy as np
import torch

own = False


def _append(name, tokens, q_heads, heads, dim, rotary, page, bits, past, neighbours=False, tree=False, columns=False):
    return dict(name=name, kind="append", tokens=tokens, q_heads=q_heads, heads=heads, dim=dim, rotary=rotary, page=page, bits=bits, past=past,
                neighbours=neighbours, tree=tree, columns=columns)


def _tree(name, batch, new, past, heads, kv_heads, dim, page, bits, ragged=False, columns=False):
    return dict(name=name, kind="tree", batch=batch, new=new, past=past, heads=heads, kv_heads=kv_heads, dim=dim, page=page, bits=bits,
                ragged=ragged, columns=columns)


def _check(name, batch, nodes, vocab, ragged=False, greedy=False):
    return dict(name=name, kind="check", batch=batch, nodes=nodes, vocab=vocab, ragged=ragged, greedy=greedy)


def _keep(name, layers, batch, nodes, kept, past, heads, dim, page, bits):
    return dict(name=name, kind="keep", layers=layers, batch=batch, nodes=nodes, kept=kept, past=past, heads=heads, dim=dim, page=page, bits=bits)


def listed():
    return [
        # the waiting token and seven nodes of a 125M-parameter model, as a product with eight vectors leaves them: latency is all there is
        _append("append 8 tokens", 8, 12, 12, 64, 64, 16, 16, 500, tree=True, columns=True),
        # a tree of 63 nodes far into a text, a model with wide heads of which a quarter is rotated in neighbouring pairs, 8 bits
        _append("append 64 tokens 8 bits", 64, 16, 16, 256, 64, 64, 8, 100000, neighbours=True, tree=True),
        # a long prompt of a 70B model with grouped heads, kept in 4 bits
        _append("append 8191 tokens 4 bits", 8191, 64, 8, 128, 128, 64, 4, 0),
        # the waiting token and seven nodes of a 125M-parameter model early in a text
        _tree("tree 1x8 of 200", 1, 8, 192, 12, 12, 64, 16, 16, columns=True),
        # small trees of 16 sequences of all lengths, grouped heads, 8 bits
        _tree("tree 16x16 of 8192 8 bits", 16, 16, 8176, 64, 8, 128, 64, 8, ragged=True),
        # a tree of 63 nodes of a 13B model at the end of a long text
        _tree("tree 1x64 of 32768", 1, 64, 32704, 40, 40, 128, 256, 16),
        # odd trees of eight sequences, a 2.7B model's heads of 80, 4 bits
        _tree("tree 8x49 of 2000 4 bits", 8, 49, 1951, 32, 32, 80, 32, 4, ragged=True),
        # one large tree of a model with grouped heads
        _tree("tree 1x257 of 16000", 1, 257, 15743, 32, 8, 128, 64, 16),
        # one tree of the size that a single text is drafted with
        _check("check 1x26 of 32000", 1, 26, 32000),
        # trees of up to 63 nodes of 32 sequences, a large vocabulary
        _check("check 32x63 of 128256", 32, 63, 128256, ragged=True),
        # an accepted path of a 13B model, its 40 layers
        _keep("keep 1x5 of 26, 40 layers", 40, 1, 26, 5, 300, 40, 128, 16, 16),
        # those of 32 sequences of a 70B model with grouped heads, 32 layers, 4 bits
        _keep("keep 32x4 of 63, 32 layers 4 bits", 32, 32, 63, 4, 300, 8, 128, 64, 4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.34 or v < 64 else v // 64 * 64     # model sizes are mostly multiples of 64


_HEADS = [(12, 12, 64), (32, 32, 128), (40, 40, 128), (64, 8, 128), (32, 32, 80), (16, 2, 96), (8, 1, 256), (24, 8, 64)]
_PAGES = [16, 32, 64, 128, 256]


def draw(rng):
    kind = rng.choice(["append", "append", "tree", "tree", "tree", "check", "keep"])
    if kind == "append":
        q_heads, heads, dim = rng.choice(_HEADS)
        rotary = rng.choice([dim, dim, dim, dim // 2, dim // 4])
        c = _append("", min(_log_int(rng, 1, 8192), 8191 * 72 * 128 // ((q_heads + heads) * dim)), q_heads, heads, dim, rotary,
                    rng.choice(_PAGES), rng.choice([16, 8, 4]), 0 if rng.random() < 0.2 else _log_int(rng, 1, 1000000), rng.random() < 0.3,
                    rng.random() < 0.5, rng.random() < 0.3)
    elif kind == "tree":
        heads, kv_heads, dim = rng.choice(_HEADS)
        c = _tree("", _log_int(rng, 1, 32), _log_int(rng, 2, 257), 0 if rng.random() < 0.1 else _log_int(rng, 1, 32768), heads, kv_heads, dim,
                  rng.choice(_PAGES), rng.choice([16, 8, 4]), rng.random() < 0.5, rng.random() < 0.3)
        most = 64 * 32768 * 40 * 128
        while c["batch"] * c["new"] * (c["past"] + c["new"]) * heads * dim > most or c["batch"] * (c["past"] + c["new"]) * kv_heads * dim * 4 > 600e6:
            if c["batch"] > 1:
                c["batch"] //= 2
            elif c["past"] > c["new"]:
                c["past"] = c["past"] * 2 // 3
            else:
                c["new"] = c["new"] * 2 // 3
    elif kind == "check":
        c = _check("", _log_int(rng, 1, 32), _log_int(rng, 1, 63), _size(rng, 1000, 128256), rng.random() < 0.5, rng.random() < 0.25)
    else:
        _, heads, dim = rng.choice(_HEADS)
        kept = rng.randint(1, 8)
        layers, batch = _log_int(rng, 1, 48), _log_int(rng, 1, 32)
        while layers * batch * kept * heads * dim > 32 * 32 * 4 * 8 * 128:
            layers, batch, kept = max(1, layers * 3 // 4), max(1, batch * 3 // 4), max(1, kept - 1)
        c = _keep("", layers, batch, _log_int(rng, 2 * kept + 1, 64), kept, _log_int(rng, 1, 300), heads, dim, rng.choice(_PAGES[:3]),
                  rng.choice([16, 8, 4]))
    del c["name"]
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------------------------

def _lengths(case):
    """New tokens and tokens in all of each sequence: the same for every seed."""
    b, r = case["batch"], random.Random(str(sorted(case.items(), key=str)))
    if not case["ragged"]:
        return [case["new"]] * b, [case["past"] + case["new"]] * b
    new = [case["new"]] + [max(1, round(case["new"] * r.uniform(0.1, 1))) for _ in range(b - 1)]
    past = [case["past"]] + [round(case["past"] * r.uniform(0.1, 1)) for _ in range(b - 1)]
    return new, [n + p for n, p in zip(new, past)]


def _generator(seed, k):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + k)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _activations(g, tokens, heads, dim, columns, spread=None):
    """(tokens, heads, dim) FP16; `columns`: as a view of the (heads * dim, tokens) that a product with several vectors leaves."""
    x = _normal(g, tokens, heads, dim)
    if spread is not None:
        x *= spread
    x = x.half()
    return x.reshape(tokens, heads * dim).t().contiguous().t().reshape_as(x) if columns else x


def _columns(tokens, heads, dim, columns):
    if columns:
        return torch.empty((heads * dim, tokens), dtype=torch.float16, device="cuda").t().view(tokens, heads, dim)
    return torch.empty((tokens, heads, dim), dtype=torch.float16, device="cuda")


def _channels(g, heads, dim):
    """Keys of real models have a few channels that are much larger than the rest."""
    return 1 + 3 * (torch.rand((heads, dim), generator=g, device="cuda") < 0.04).float()


def _encode(x, bits):
    """Codes and steps of (..., dim) values in 32 bits: what the cache holds in 8 and 4 bits."""
    x = torch.nan_to_num(x, 0.0, 65504.0, -65504.0).clamp(-65504.0, 65504.0)
    if bits == 8:
        most = x.abs().amax(-1)
        step = most / 127
        inv = torch.where(most > 0, 127 / most, torch.zeros_like(most))
        return torch.clamp(torch.round(x * inv[..., None]), -127, 127).to(torch.int8), step
    low, high = x.amin(-1).half(), x.amax(-1)
    step = (torch.clamp(high - low.float(), min=0) / 15).half()
    inv = torch.where(step > 0, 1 / step.float(), torch.zeros_like(high))
    code = torch.clamp(torch.round((x - low.float()[..., None]) * inv[..., None]), 0, 15).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.stack([step, low], -1)


def _decode(code, step, bits, wide=torch.float32):
    if bits == 16:
        return code.to(wide)
    if bits == 8:
        return code.to(wide) * step.to(wide)[..., None]
    code = torch.stack([code & 15, code >> 4], -1).flatten(-2).to(wide)
    return code * step[..., 0:1].to(wide) + step[..., 1:2].to(wide)


def _empty_cache(pages, heads, page, dim, bits):
    if bits == 16:
        make = lambda: (torch.zeros((pages, heads, page, dim), dtype=torch.float16, device="cuda"), None)           # noqa: E731
    elif bits == 8:
        make = lambda: (torch.zeros((pages, heads, page, dim), dtype=torch.int8, device="cuda"),                    # noqa: E731
                        torch.zeros((pages, heads, page), dtype=torch.float32, device="cuda"))
    else:
        make = lambda: (torch.zeros((pages, heads, page, dim // 2), dtype=torch.uint8, device="cuda"),              # noqa: E731
                        torch.zeros((pages, heads, page, 2), dtype=torch.float16, device="cuda"))
    return make() + make()


def _filled(g, pages, heads, page, dim, bits, spread=None):
    """A cache's codes and steps of random values, a few pages at a time: the values in 32 bits are larger than the cache."""
    parts = []
    for p in range(0, pages, 256):
        x = _normal(g, min(256, pages - p), heads, page, dim)
        x = (x if spread is None else x * spread).half()
        parts.append((x, None) if bits == 16 else _encode(x.float(), bits))
    return tuple(None if x[0] is None else torch.cat(x) for x in zip(*parts))


def _parents(rng, nodes):
    """A random tree, its nodes in the order of their levels: each node's parent among those before it, -1 for the token before the tree."""
    return [-1 if i == 0 else int(rng.integers(max(-1, i // 4 - 3), max(0, (i + 1) // 2))) for i in range(nodes)]


def _tables(rng, need, extra=3):
    """A page table for sequences that need so many pages each, of pages in no order; how many pages there are."""
    pages = sum(need) + extra
    order = rng.permutation(pages)
    table, at = np.zeros((len(need), max(need)), np.int32), 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    return torch.from_numpy(table).cuda(), pages


def _prepare_append(case, seed):
    t, hq, h, d, page, bits = (case[k] for k in ("tokens", "q_heads", "heads", "dim", "page", "bits"))
    g = _generator(seed, 1)
    pages = 2 * (-(-t // page)) + 3                          # other sequences have the rest
    table = torch.randperm(pages, generator=g, device="cuda")[:-(-t // page)]
    at = torch.arange(t, device="cuda")
    pairs = case["rotary"] // 2
    s = dict(q=_activations(g, t, hq, d, case["columns"]), k=_activations(g, t, h, d, case["columns"], _channels(g, h, d)),
             v=_activations(g, t, h, d, case["columns"]), q_out=_columns(t, hq, d, case["columns"]),
             slots=table[at // page] * page + at % page, position=(case["past"] + (at // 4 if case["tree"] else at)).int(),
             frequency=10000.0 ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs), neighbours=case["neighbours"],
             bits=bits, cache=_empty_cache(pages, h, page, d, bits))
    if bits < 16:
        s.update(k_back=_columns(t, h, d, False), v_back=_columns(t, h, d, False))
    if own:
        from paper_2507_12205_amd import device as D
        k, ks, v, vs = s["cache"]
        s.update(D=D, kv=D.KvCache(k, v, ks, vs))
    return s


def _prepare_tree(case, seed):
    b, h, hk, d, page, bits = (case[k] for k in ("batch", "heads", "kv_heads", "dim", "page", "bits"))
    new, total = _lengths(case)
    g, rng = _generator(seed, 2), np.random.default_rng([seed, 2])
    table, pages = _tables(rng, [-(-n // page) for n in total])
    k, ks = _filled(g, pages, hk, page, d, bits, _channels(g, hk, d)[None, :, None, :])
    v, vs = _filled(g, pages, hk, page, d, bits)
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    tokens, words = int(start[-1]), -(-max(new) // 32)
    seen = np.zeros((tokens, words), np.uint32)              # bit i of a token: it sees the sequence's i-th new token
    for i, n in enumerate(new):
        rows = seen[start[i]:start[i + 1]]
        rows[0, 0] = 1                                       # the waiting token, and the tree below it
        for j, p in enumerate(_parents(rng, n - 1), 1):
            rows[j] = rows[p + 1]
            rows[j, j // 32] |= np.uint32(1) << np.uint32(j % 32)
    s = dict(q=_activations(g, tokens, h, d, case["columns"]), out=_columns(tokens, h, d, case["columns"]), cache=(k, ks, v, vs), bits=bits,
             start=torch.from_numpy(start).cuda(), total=torch.tensor(total, dtype=torch.int32, device="cuda"),
             table=table, seen=torch.from_numpy(seen.view(np.int32)).cuda(), most_new=max(new), most=max(total), page=page, scale=1 / math.sqrt(d))
    if own:
        from paper_2507_12205_amd import device as D
        s.update(D=D, kv=D.KvCache(k, v, ks, vs))
        s["work"] = D.attention_workspace(s["kv"], s["q"], b, s["most_new"], table.shape[1] * page)
    return s


def _prepare_check(case, seed):
    b, k, n = case["batch"], case["nodes"], case["vocab"]
    g, rng = _generator(seed, 3), np.random.default_rng([seed, 3])
    p = torch.softmax(6 * _normal(g, b, k + 1, n), -1)
    parent = np.array([_parents(rng, k) for _ in range(b)], np.int64).reshape(b, k)
    rank = np.array([[int((parent[i, :j] == parent[i, j]).sum()) for j in range(k)] for i in range(b)]).reshape(b, k)
    rows = torch.arange(b, device="cuda")[:, None]
    parent = torch.from_numpy(parent).cuda()
    likely = torch.topk(p, 64).indices                       # a draft model that ranks the candidates as the target does
    drafted = likely[rows, parent + 1, torch.from_numpy(rank % 64).cuda()].int()
    if case["greedy"]:
        p = torch.zeros_like(p).scatter_(2, likely[..., :1], 1.0)
    s = dict(p=p, drafted=drafted, parent=parent.int(), u=torch.rand((b, k + 1), generator=g, device="cuda"),
             count=torch.randint(0, k + 1, (b,), generator=g, device="cuda", dtype=torch.int32) if case["ragged"] else None,
             tokens=torch.empty((b, k + 1), dtype=torch.int32, device="cuda"), path=torch.empty((b, k), dtype=torch.int32, device="cuda"),
             accepted=torch.empty((b,), dtype=torch.int32, device="cuda"))
    if own:
        from paper_2507_12205_amd import device as D
        s["D"] = D
    return s


def _prepare_keep(case, seed):
    b, nodes, kept, page = case["batch"], case["nodes"], case["kept"], case["page"]
    g, rng = _generator(seed, 4), np.random.default_rng([seed, 4])
    table, pages = _tables(rng, [-(-(case["past"] + nodes) // page)] * b)
    shape = (pages, case["heads"], page, case["dim"], case["bits"])
    # the likeliest candidates were refused: every row that is kept lies behind the places of all of them
    path = np.stack([np.sort(rng.choice(np.arange(kept, nodes), kept, replace=False)) for _ in range(b)])
    path = np.concatenate([path, np.full((b, nodes - kept), -1)], 1).astype(np.int32)
    # all layers' caches lie in one allocation for each of their tensors
    whole = [torch.stack(x) for x in zip(*([t for t in _filled(g, *shape) + _filled(g, *shape) if t is not None] for _ in range(case["layers"])))]
    s = dict(whole=whole, table=table, page=page,
             first=torch.from_numpy(rng.integers(0, case["past"] + 1, b).astype(np.int32)).cuda(), path=torch.from_numpy(path).cuda(),
             accepted=torch.full((b,), kept, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2507_12205_amd import device as D
        s.update(D=D, kv=D.KvCaches([D.KvCache(t[0], t[1]) if len(t) == 2 else D.KvCache(t[0], t[2], t[1], t[3]) for t in zip(*whole)]))
    return s


def prepare(case, seed):
    s = {"append": _prepare_append, "tree": _prepare_tree, "check": _prepare_check, "keep": _prepare_keep}[case["kind"]](case, seed)
    s["kind"] = case["kind"]
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------------------

def _own_append(s):
    s["D"].kv_append(s["kv"], s["k"], s["v"], s["slots"], s["position"], s["frequency"], s["q"], s["q_out"], s["neighbours"])
    if s["bits"] == 16:
        return [s["q_out"], s["cache"][0], s["cache"][2]]
    return [s["q_out"], *s["D"].kv_read(s["kv"], s["slots"], s["k_back"], s["v_back"])]       # what the codes stand for


def _own_tree(s):
    return s["D"].attention_tree(s["kv"], s["q"], s["out"], s["start"], s["total"], s["table"], s["seen"], s["most_new"], s["scale"], s["work"])


def _own_check(s):
    return s["D"].verify_tree(s["p"], s["drafted"], s["parent"], s["u"], s["tokens"], s["path"], s["accepted"], s["count"])


def _own_keep(s):
    s["D"].kv_keep(s["kv"], s["first"], s["path"], s["accepted"], s["table"])
    return s["whole"]


def _rotate(x, cos, sin, neighbours):
    """(tokens, heads, dim) in the type of cos and sin, (tokens, 1, pairs): the pairs (a, b) become (a cos - b sin, a sin + b cos)."""
    pairs = cos.shape[-1]
    x = x.to(cos.dtype)
    if neighbours:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., 2 * pairs:]], -1)


def _plain_append(s):
    angle = (s["position"].double()[:, None] * s["frequency"])[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()                 # (32 bits would lose the angles of far positions)
    q, k = (_rotate(s[name], cos, sin, s["neighbours"]) for name in ("q", "k"))
    kc, ks, vc, vs = s["cache"]
    page = kc.shape[2]
    at, off, back = s["slots"] // page, s["slots"] % page, []
    for x, code, step in ((k, kc, ks), (s["v"].float(), vc, vs)):
        if s["bits"] == 16:
            code[at, :, off] = x.half()
            back.append(code)
        else:
            c, st = _encode(x, s["bits"])
            code[at, :, off] = c
            step[at, :, off] = st
            back.append(_decode(code[at, :, off], step[at, :, off], s["bits"]).half())
    return [q.half(), *back]


def _plain_tree(s):
    q, start, total, table, page = s["q"].float(), s["start"].long(), s["total"].long(), s["table"].long(), s["page"]
    k, ks, v, vs = s["cache"]
    b, hk, h = table.shape[0], k.shape[1], q.shape[1]
    new = start[1:] - start[:-1]
    t = torch.arange(s["most_new"], device="cuda")
    j = torch.arange(s["most"], device="cuda")
    row = torch.minimum(start[:-1, None] + t, start[1:, None] - 1)                 # short trees repeat their last token
    qp = q[row].permute(0, 2, 1, 3).reshape(b, hk, -1, q.shape[2])                 # (sequence, head of the cache, heads of its group x tokens, dim)
    pages, off = table[:, j // page], j % page

    def gather(code, step):
        return _decode(code[pages, :, off], None if step is None else step[pages, :, off], s["bits"]).permute(0, 2, 1, 3)
    scores = qp @ gather(k, ks).transpose(2, 3).contiguous() * s["scale"]
    node = j - (total - new)[:, None]                                              # (sequence, key): which of the new tokens it is
    bits = (s["seen"][row][..., t // 32] >> (t % 32).int()) & 1                    # (sequence, token, new token)
    index = node.clamp(0, len(t) - 1)[:, None].expand(-1, len(t), -1)
    seen = (node < 0)[:, None] | ((node < new[:, None])[:, None] & (bits.gather(2, index) != 0))
    scores = scores.view(b, hk, h // hk, len(t), len(j)).masked_fill_(~seen[:, None, None], float("-inf"))
    scores = torch.exp(scores - scores.amax(-1, keepdim=True))
    scores = scores / scores.sum(-1, keepdim=True)
    o = (scores.view(b, hk, -1, len(j)) @ gather(v, vs).contiguous()).view(b, h, len(t), -1).permute(0, 2, 1, 3)
    return o[t < new[:, None]].half()


def _plain_check(s):
    p, x, parent, u = s["p"], s["drafted"].long(), s["parent"].long(), s["u"].double()
    b, k = x.shape
    rows, minus = torch.arange(b, device="cuda"), torch.full((b,), -1, dtype=torch.long, device="cuda")
    count = torch.full((b,), k, device="cuda") if s["count"] is None else s["count"].long()
    px = p[rows[:, None], parent + 1, x].double()
    # whole numbers, decided by where a value passes a bound: in 64 bits, as any order of additions then decides alike
    at, left, n = minus, torch.ones(b, dtype=torch.float64, device="cuda"), torch.zeros(b, dtype=torch.long, device="cuda")
    refused = torch.zeros((b, k), dtype=torch.bool, device="cuda")
    path = torch.full((b, k + 1), -1, dtype=torch.int32, device="cuda")
    for i in range(k):
        again = (refused & (parent == at[:, None]) & (x == x[:, i:i + 1])).any(1)
        asked = (parent[:, i] == at) & (i < count) & ~again
        ok = asked & (u[:, i] * left < px[:, i])
        refused[:, i] = asked & ~ok
        left = torch.where(ok, torch.ones_like(left), torch.where(asked, left - px[:, i].clamp(min=0), left))
        path.scatter_(1, torch.where(ok, n, torch.full_like(n, k))[:, None], torch.full((b, 1), i, dtype=torch.int32, device="cuda"))
        at = torch.where(ok, torch.full_like(at, i), at)
        n = n + ok
    path = torch.where(torch.arange(k, device="cuda") < n[:, None], path[:, :k], torch.full_like(path[:, :k], -1))
    w = p[rows, at + 1].double()
    gone = refused & (parent == at[:, None])
    hit = torch.zeros((b, w.shape[1] + 1), dtype=torch.bool, device="cuda")
    hit.scatter_(1, torch.where(gone, x, torch.full_like(x, w.shape[1])), True)
    rest = w.masked_fill(hit[:, :-1], 0.0)
    w = torch.where((rest.sum(1) > 0)[:, None], rest, w)                           # (nothing is left where all of it was drafted)
    c = torch.cumsum(w, 1)
    token = (c <= u[:, k:] * c[:, -1:]).sum(1)
    last = w.shape[1] - 1 - torch.flip(w > 0, [1]).int().argmax(1)
    token = torch.minimum(token, last).int()
    j = torch.arange(k + 1, device="cuda")
    named = torch.cat([x.int().gather(1, path.long().clamp(min=0)), token[:, None]], 1)
    tokens = torch.where(j < n[:, None], named, torch.where(j == n[:, None], token[:, None], torch.full_like(named, -1)))
    return tokens, path, n.int()


def _plain_keep(s):
    table, page, path = s["table"].long(), s["page"], s["path"].long()
    i = torch.arange(path.shape[1], device="cuda")
    to = s["first"].long()[:, None] + i
    at = torch.where(i < s["accepted"][:, None], s["first"].long()[:, None] + path, to)        # (the others stay where they are)
    src, dst = (torch.gather(table, 1, x // page) for x in (at, to))
    for tensor in s["whole"]:
        tensor[:, dst, :, to % page] = tensor[:, src, :, at % page]
    return s["whole"]


def run(state):
    kind = state["kind"]
    if own:
        return {"append": _own_append, "tree": _own_tree, "check": _own_check, "keep": _own_keep}[kind](state)
    return {"append": _plain_append, "tree": _plain_tree, "check": _plain_check, "keep": _plain_keep}[kind](state)


# ---- what a pass cannot do without, and what it returns in 64 bits --------------------------------------------------------------------

def _row_bytes(dim, bits):
    return dim * bits / 8 + (0 if bits == 16 else 4)


def work(case):
    if case["kind"] == "append":
        t, q, rows = case["tokens"], case["tokens"] * case["q_heads"], 2 * case["tokens"] * case["heads"]
        # queries read and written, keys and values read, their rows written; codes read back, and their values written
        back = 0 if case["bits"] == 16 else _row_bytes(case["dim"], case["bits"]) + 2 * case["dim"]
        return {"bytes": 4.0 * q * case["dim"] + rows * (2 * case["dim"] + _row_bytes(case["dim"], case["bits"]) + back) + 12 * t,
                "flops": 3.0 * (q + rows / 2) * case["rotary"] + (0 if case["bits"] == 16 else 4.0 * rows * case["dim"])}
    if case["kind"] == "tree":
        new, total = _lengths(case)
        pairs = sum(n * (t - n) + n for n, t in zip(new, total))                   # what came before, and each token itself
        return {"bytes": 2 * sum(total) * case["kv_heads"] * _row_bytes(case["dim"], case["bits"]) + 4 * sum(new) * case["heads"] * case["dim"],
                "flops": 4.0 * pairs * case["heads"] * case["dim"]}
    if case["kind"] == "check":
        return {"bytes": case["batch"] * (4.0 * case["vocab"] + 24 * case["nodes"]), "flops": 2.0 * case["batch"] * case["vocab"]}
    rows = 2 * case["layers"] * case["batch"] * case["kept"] * case["heads"]
    return {"bytes": 2.0 * rows * _row_bytes(case["dim"], case["bits"]) + 8 * case["batch"] * case["kept"], "flops": 0.0}


def _exact_values(x, bits):
    """What the cache stands for, in 64 bits, from the definition of its steps."""
    if bits == 16:
        return x
    if bits == 8:
        step = x.abs().max(dim=-1, keepdim=True).values / 127
        return torch.where(step > 0, torch.round(x / step.clamp(min=1e-300)), 0.0) * step
    low = x.min(dim=-1, keepdim=True).values.half().double()
    step = ((x.max(dim=-1, keepdim=True).values - low).clamp(min=0) / 15).half().double()
    return low + step * torch.where(step > 0, torch.round((x - low) / step.clamp(min=1e-300)).clamp(0, 15), 0.0)


def _exact_append(case, s):
    """A pair as a complex number times exp(i angle)."""
    pairs = case["rotary"] // 2
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda").expand(case["tokens"], pairs),
                       torch.outer(s["position"].double(), s["frequency"]))[:, None]

    def turned(x):
        y = x.double().clone()
        part = y[..., :2 * pairs].unflatten(-1, (pairs, 2) if case["neighbours"] else (2, pairs))
        part = part if case["neighbours"] else part.transpose(-1, -2)
        z = torch.view_as_real(torch.complex(part[..., 0].contiguous(), part[..., 1].contiguous()) * turn)
        y[..., :2 * pairs] = (z if case["neighbours"] else z.transpose(-1, -2)).flatten(-2)
        return y
    k, v = _exact_values(turned(s["k"]), case["bits"]), _exact_values(s["v"].double(), case["bits"])
    if case["bits"] < 16:
        return [turned(s["q"]), k, v]
    out = []
    for x, cache in ((k, s["cache"][0]), (v, s["cache"][2])):
        whole = torch.zeros(cache.shape, dtype=torch.float64, device="cuda")
        whole.transpose(1, 2)[s["slots"] // case["page"], s["slots"] % case["page"]] = x
        out.append(whole)
    return [turned(s["q"]), *out]


def _exact_keep(case, s):
    """One row after the other; codes are whole numbers, which have to be equal."""
    first, path, table, page, out = s["first"].tolist(), s["path"].tolist(), s["table"].tolist(), case["page"], []
    for tensor in s["whole"]:
        x = tensor.double() if tensor.dtype.is_floating_point else None
        for b in range(case["batch"] if x is not None else 0):
            for i in range(case["kept"]):
                at, to = first[b] + path[b][i], first[b] + i
                x[:, table[b][to // page], :, to % page] = x[:, table[b][at // page], :, at % page].clone()
        out.append(x)
    return out


def exact(case, seed):
    if case["kind"] == "check":
        return None                                          # whole numbers: they have to be equal
    s = prepare(case, seed)
    if case["kind"] == "keep":
        return _exact_keep(case, s)
    if case["kind"] == "append":
        return _exact_append(case, s)
    new, total = _lengths(case)
    group, out, at = case["heads"] // case["kv_heads"], [], 0
    k, ks, v, vs = s["cache"]
    words = s["seen"].cpu().numpy().view(np.uint32)
    for i in range(case["batch"]):
        where = s["table"][i, :-(-total[i] // case["page"])].long()

        def sequence(code, step):
            x = _decode(code[where], None if step is None else step[where], case["bits"], torch.float64)
            return x.transpose(1, 2).reshape(-1, case["kv_heads"], case["dim"])[:total[i]]
        kk, vv = sequence(k, ks), sequence(v, vs)
        q = s["q"][at:at + new[i]].double()
        hidden = np.zeros((new[i], total[i]), bool)
        for t in range(new[i]):
            for j in range(new[i]):
                hidden[t, total[i] - new[i] + j] = not (int(words[at + t, j // 32]) >> (j % 32)) & 1
        hidden = torch.from_numpy(hidden).cuda()
        o = torch.empty((new[i], case["heads"], case["dim"]), dtype=torch.float64, device="cuda")
        for h in range(case["heads"]):
            a = (q[:, h].contiguous() @ kk[:, h // group].t().contiguous()) / math.sqrt(case["dim"])
            o[:, h] = torch.softmax(a.masked_fill_(hidden, -math.inf), -1) @ vv[:, h // group].contiguous()
        out.append(o)
        at += new[i]
    return torch.cat(out)
