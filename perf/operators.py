"""The operators around the products of a pruned model that is being served, as timed cases: a product with its epilogue, the paged
cache of keys and values, the attention of new tokens over it, and the check of drafted tokens.

With `own` false they are computed in plain torch operations; with `own` true by the calls a serving program makes of this library.

A case is a dict:
  kind "product"    y = act(W x + bias) * gate + residual for a pruned W
       m, n, density, bits (of a delta index), fp32, nb (vectors), act ("none", "relu", "gelu", "silu"), bias, gate, residual (whether there)
  kind "cache"      `tokens` new keys and values written into their places of a paged cache, and read back
       tokens, heads (of keys and values), dim, page (tokens), bits (16, 8 or 4 for a cached value), columns
  kind "attention"  attention of the new tokens of `batch` sequences over the cache that holds them and what came before
       batch, new (most new tokens of a sequence), past (most tokens before them), ragged (lengths from a tenth of that up),
       heads, kv_heads, dim, page, bits, columns (activations as the products leave them: one column per token)
  kind "verify"     `drafts` drafted tokens of `batch` sequences against the target's probabilities over `vocab` tokens
       batch, drafts, vocab, ragged (fewer drafts in some sequences), greedy (drafts without probabilities of their own)
"""
import math
import random

import numpy as np
import torch

own = False


def _product(name, m, n, density, bits, act, bias, gate, residual, fp32=False, nb=1):
    return dict(name=name, kind="product", m=m, n=n, density=density, bits=bits, fp32=fp32, nb=nb, act=act, bias=bias, gate=gate,
                residual=residual)


def _cache(name, tokens, heads, dim, page, bits, columns=False):
    return dict(name=name, kind="cache", tokens=tokens, heads=heads, dim=dim, page=page, bits=bits, columns=columns)


def _attention(name, batch, new, past, heads, kv_heads, dim, page, bits, ragged=False, columns=False):
    return dict(name=name, kind="attention", batch=batch, new=new, past=past, heads=heads, kv_heads=kv_heads, dim=dim, page=page, bits=bits,
                ragged=ragged, columns=columns)


def _verify(name, batch, drafts, vocab, ragged=False, greedy=False):
    return dict(name=name, kind="verify", batch=batch, drafts=drafts, vocab=vocab, ragged=ragged, greedy=greedy)


def listed():
    return [
        # attention's output projection of a 125M-parameter model, one token: the launch is all there is
        _product("product 768x768", 768, 768, 0.5, 4, "none", True, False, True),
        # the gated MLP product of a 13B model at 70 % sparsity, one token
        _product("product gated 13824x5120", 13824, 5120, 0.3, 4, "silu", True, True, False),
        # a model kept in FP32, odd sizes, two tokens, everything an epilogue has
        _product("product fp32 2x 2999x5003", 2999, 5003, 0.3, 8, "gelu", True, True, True, fp32=True, nb=2),
        # one decoding step of four sequences of a 7B model, keys and values as the products leave them
        _cache("cache 4 tokens 8 bits", 4, 32, 128, 16, 8, columns=True),
        # a long prompt of a 70B model with grouped heads, kept in 4 bits
        _cache("cache 8191 tokens 4 bits", 8191, 8, 128, 64, 4),
        # one token of a 125M-parameter model early in a text
        _attention("attention 1 of 200", 1, 1, 199, 12, 12, 64, 16, 16),
        # a decoding step of 16 sequences of all lengths, grouped heads, 8 bits
        _attention("attention 16x1 of 8192 8 bits", 16, 1, 8191, 64, 8, 128, 64, 8, ragged=True),
        # eight drafted tokens of a 13B model at the end of a long text, columns as the products have them
        _attention("attention 8 of 32768", 1, 8, 32760, 40, 40, 128, 256, 16, columns=True),
        # a chunk of a long prompt of a 7B model
        _attention("attention 2048 of 4096", 1, 2048, 2048, 32, 32, 128, 64, 16),
        # chunks of all lengths of several prompts, a 2.7B model's heads of 80, 4 bits, odd lengths
        _attention("attention 5x333 of 3000 4 bits", 5, 333, 2667, 32, 32, 80, 32, 4, ragged=True),
        # four drafted tokens of one sequence
        _verify("verify 1x4 of 32000", 1, 4, 32000),
        # up to seven drafted tokens of 32 sequences, a large vocabulary
        _verify("verify 32x7 of 128256", 32, 7, 128256, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.34 or v < 64 else v // 64 * 64     # model sizes are mostly multiples of 64


def draw(rng):
    kind = rng.choice(["product", "product", "cache", "attention", "attention", "attention", "verify"])
    if kind == "product":
        fp32, nb = rng.random() < 0.3, rng.choice([1, 1, 2, 4, 8])
        m, n = _size(rng, 512, 13824), _size(rng, 512, 13824)
        if nb > 1:
            n = min(n, 8192 if fp32 else 13824)             # two vectors and their partial sums have to fit a compute unit's memory
        c = _product("", m, n, round(rng.uniform(0.1, 0.5), 3), rng.choice([4, 8]), rng.choice(["none", "relu", "gelu", "silu"]),
                     rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.6, fp32, nb)
        while c["m"] * c["n"] * c["density"] > 13824 * 5120 * 0.3:
            c["m"] = max(256, c["m"] * 3 // 4)
    elif kind == "cache":
        heads, dim = rng.choice([(12, 64), (32, 128), (40, 128), (8, 128), (32, 80), (2, 256)])
        c = _cache("", min(_log_int(rng, 1, 8192), 8192 * 8 * 128 // (heads * dim)), heads, dim, rng.choice([16, 32, 64, 128, 256]),
                   rng.choice([16, 8, 4]), rng.random() < 0.3)
    elif kind == "attention":
        heads, kv_heads, dim = rng.choice([(12, 12, 64), (32, 32, 128), (40, 40, 128), (64, 8, 128), (32, 32, 80), (16, 2, 96), (8, 1, 256),
                                           (24, 8, 64)])
        new = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 9, 2048)])
        past = 0 if rng.random() < 0.1 else _log_int(rng, 1, 32768)
        c = _attention("", _log_int(rng, 1, 32), new, past, heads, kv_heads, dim, rng.choice([16, 32, 64, 128, 256]), rng.choice([16, 8, 4]),
                       rng.random() < 0.5, rng.random() < 0.3)
        most = 2 * 4 * 2048 * (2048 + 1024) * 32 * 128 // 3
        while c["batch"] * c["new"] * (c["past"] + c["new"]) * heads * dim * 4 > most or c["batch"] * (c["past"] + c["new"]) * kv_heads * dim * 4 > 600e6:
            if c["batch"] > 1:
                c["batch"] //= 2
            elif c["past"] > c["new"]:
                c["past"] = c["past"] * 2 // 3
            else:
                c["new"] = c["new"] * 2 // 3
    else:
        c = _verify("", _log_int(rng, 1, 32), rng.randint(1, 7), _size(rng, 1000, 128256), rng.random() < 0.5, rng.random() < 0.25)
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
    """Codes and steps of (..., dim) values: what the cache holds in 8 and 4 bits."""
    x = torch.nan_to_num(x.float(), 0.0, 65504.0, -65504.0)
    if bits == 8:
        most = x.abs().amax(-1)
        step = most / 127
        inv = torch.where(most > 0, 127 / most, torch.zeros_like(most))
        return torch.clamp(torch.round(x * inv[..., None]), -127, 127).to(torch.int8), step
    low, high = x.amin(-1), x.amax(-1)
    step = ((high - low) / 15).half().float()
    inv = torch.where(step > 0, 1 / step, torch.zeros_like(step))
    code = torch.clamp(torch.round((x - low[..., None]) * inv[..., None]), 0, 15).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.stack([step, low], -1).half()


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


def _weights(case, seed):
    """A dense pruned matrix: every column has its own share of kept entries, a tenth of them lies in dense blocks."""
    m, n, density = case["m"], case["n"], case["density"]
    g, rng = _generator(seed, 1), np.random.default_rng([seed, m, n])
    q = rng.beta(2.0, 2.0, n).astype(np.float32)
    p = torch.from_numpy(np.clip(q / q.mean() * 0.9 * density, 0.02, 0.98)).cuda()
    keep = torch.rand((m, n), generator=g, device="cuda") < p
    blocks = int(0.1 * density * m * n / (16 * 32))
    if blocks:
        rows = torch.randint(0, m, (blocks, 16, 1), generator=g, device="cuda")
        cols = torch.randint(0, n, (blocks, 1, 32), generator=g, device="cuda")
        keep.view(-1)[(rows * n + cols).view(-1)] = True
    return _normal(g, m, n).mul_(0.02).masked_fill_(~keep, 0).to(torch.float32 if case["fp32"] else torch.float16)


def _prepare_product(case, seed):
    dt = torch.float32 if case["fp32"] else torch.float16
    m, n, nb, g = case["m"], case["n"], case["nb"], _generator(seed, 2)
    shape = (lambda r: (r,)) if nb == 1 else (lambda r: (r, nb))
    s = dict(w=_weights(case, seed), x=_normal(g, *shape(n)).to(dt), y=torch.empty(shape(m), dtype=dt, device="cuda"), act=case["act"],
             bias=(0.5 * _normal(g, m)).to(dt) if case["bias"] else None, gate=_normal(g, *shape(m)).to(dt) if case["gate"] else None,
             residual=_normal(g, *shape(m)).to(dt) if case["residual"] else None)
    if own:                                                 # the image that a serving program builds of its weights when it loads them
        import paper_2507_12205_amd as E
        from paper_2507_12205_amd import device as D
        build = E.ecspmv_build_dense_f32 if case["fp32"] else E.ecspmv_build_dense
        s.update(D=D, mat=build(s["w"].cpu().numpy(), E.make_opts(delta_bits=case["bits"])))
        D.upload(s["mat"])
    return s


def _prepare_cache(case, seed):
    t, h, d, page, bits = (case[k] for k in ("tokens", "heads", "dim", "page", "bits"))
    g = _generator(seed, 3)
    pages = 2 * (-(-t // page)) + 3                          # other sequences have the rest
    table = torch.randperm(pages, generator=g, device="cuda")[:-(-t // page)]
    at = torch.arange(t, device="cuda")
    s = dict(k=_activations(g, t, h, d, case["columns"], _channels(g, h, d)), v=_activations(g, t, h, d, case["columns"]),
             slots=table[at // page] * page + at % page, bits=bits, cache=_empty_cache(pages, h, page, d, bits),
             k_back=_columns(t, h, d, case["columns"]), v_back=_columns(t, h, d, case["columns"]))
    if own:
        from paper_2507_12205_amd import device as D
        k, ks, v, vs = s["cache"]
        s.update(D=D, kv=D.KvCache(k, v, ks, vs))
    return s


def _prepare_attention(case, seed):
    b, h, hk, d, page, bits = (case[k] for k in ("batch", "heads", "kv_heads", "dim", "page", "bits"))
    new, total = _lengths(case)
    g, rng = _generator(seed, 4), np.random.default_rng([seed, 4])
    need = [-(-n // page) for n in total]
    pages, most = sum(need) + 3, max(need)
    order = rng.permutation(pages)
    table, at = np.zeros((b, most), np.int32), 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    k_cache, v_cache = [], []
    spread = _channels(g, hk, d)[None, :, None, :]
    for p in range(0, pages, 256):                          # (a few pages at a time: the values in 32 bits are larger than the cache)
        count = min(256, pages - p)
        for to, wide in ((k_cache, spread), (v_cache, 1.0)):
            x = (_normal(g, count, hk, page, d) * wide).half()
            to.append((x, None) if bits == 16 else _encode(x, bits))
    def whole(parts):                                       # noqa: E306
        return tuple(None if x[0] is None else torch.cat(x) for x in zip(*parts))
    k, ks = whole(k_cache)
    v, vs = whole(v_cache)
    del k_cache, v_cache
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    tokens = int(start[-1])
    s = dict(q=_activations(g, tokens, h, d, case["columns"]), out=_columns(tokens, h, d, case["columns"]), cache=(k, ks, v, vs), bits=bits,
             start=torch.from_numpy(start).cuda(), total=torch.tensor(total, dtype=torch.int32, device="cuda"),
             table=torch.from_numpy(table).cuda(), most_new=max(new), most=max(total), page=page, scale=1 / math.sqrt(d))
    if own:
        from paper_2507_12205_amd import device as D
        s.update(D=D, kv=D.KvCache(k, v, ks, vs))
        s["work"] = D.attention_workspace(s["kv"], s["q"], b, s["most_new"], most * page)
    return s


def _prepare_verify(case, seed):
    b, k, n, g = case["batch"], case["drafts"], case["vocab"], _generator(seed, 5)
    logits = 2.5 * _normal(g, b, k + 1, n)
    p = torch.softmax(logits, -1)
    q = torch.softmax(logits[:, :k] + 0.7 * _normal(g, b, k, n), -1)              # a draft model that is often right
    drafted = torch.multinomial(q.view(b * k, n), 1, generator=g).view(b, k).int()
    s = dict(p=p, q=None if case["greedy"] else q, drafted=drafted, u=torch.rand((b, k + 1), generator=g, device="cuda"),
             count=torch.randint(0, k + 1, (b,), generator=g, device="cuda", dtype=torch.int32) if case["ragged"] else None,
             tokens=torch.empty((b, k + 1), dtype=torch.int32, device="cuda"), accepted=torch.empty((b,), dtype=torch.int32, device="cuda"))
    if own:
        from paper_2507_12205_amd import device as D
        s["D"] = D
    return s


def prepare(case, seed):
    s = {"product": _prepare_product, "cache": _prepare_cache, "attention": _prepare_attention, "verify": _prepare_verify}[case["kind"]](case, seed)
    s["kind"] = case["kind"]
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------------------

def _own_product(s):
    return s["D"].run_epilogue(s["mat"], s["x"], s["y"], s["bias"], s["act"], s["gate"], s["residual"])


def _own_cache(s):
    s["D"].kv_write(s["kv"], s["k"], s["v"], s["slots"])
    return s["D"].kv_read(s["kv"], s["slots"], s["k_back"], s["v_back"])


def _own_attention(s):
    return s["D"].attention(s["kv"], s["q"], s["out"], s["start"], s["total"], s["table"], s["most_new"], s["scale"], s["work"])


def _own_verify(s):
    return s["D"].verify(s["p"], s["q"], s["drafted"], s["u"], s["tokens"], s["accepted"], s["count"])


def _act(t, name):
    if name == "relu":
        return torch.clamp(t, min=0)
    if name == "silu":
        return t / (1 + torch.exp(-t))
    if name == "gelu":
        return 0.5 * t * (1 + torch.erf(t / math.sqrt(2)))
    return t


def _plain_product(s):
    y = s["w"].float() @ s["x"].float()
    if s["bias"] is not None:
        y = y + (s["bias"].float() if y.dim() == 1 else s["bias"].float()[:, None])
    y = _act(y, s["act"])
    if s["gate"] is not None:
        y = y * s["gate"].float()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["y"].dtype)


def _plain_cache(s):
    k, ks, v, vs = s["cache"]
    page = k.shape[2]
    at, off, back = s["slots"] // page, s["slots"] % page, []
    for x, code, step in ((s["k"], k, ks), (s["v"], v, vs)):
        if s["bits"] == 16:
            code[at, :, off] = x
            back.append(code[at, :, off])
        else:
            c, st = _encode(x, s["bits"])
            code[at, :, off] = c
            step[at, :, off] = st
            back.append(_decode(code[at, :, off], step[at, :, off], s["bits"]).half())
    return back


def _plain_attention(s):
    q, start, total, table, page = s["q"].float(), s["start"].long(), s["total"].long(), s["table"].long(), s["page"]
    k, ks, v, vs = s["cache"]
    b, hk, h = table.shape[0], k.shape[1], q.shape[1]
    new = start[1:] - start[:-1]
    t = torch.arange(s["most_new"], device="cuda")
    j = torch.arange(s["most"], device="cuda")
    row = torch.minimum(start[:-1, None] + t, start[1:, None] - 1)                 # short chunks repeat their last token
    qp = q[row].permute(0, 2, 1, 3).reshape(b, hk, -1, q.shape[2])                 # (sequence, head of the cache, heads of its group x tokens, dim)
    pages, off = table[:, j // page], j % page

    def gather(code, step):
        return _decode(code[pages, :, off], None if step is None else step[pages, :, off], s["bits"]).permute(0, 2, 1, 3)
    scores = qp @ gather(k, ks).transpose(2, 3).contiguous() * s["scale"]
    seen = j <= (total[:, None, None] - new[:, None, None] + t[None, :, None])     # (sequence, token, key)
    scores = scores.view(b, hk, h // hk, len(t), len(j)).masked_fill_(~seen[:, None, None], float("-inf"))
    scores = torch.exp(scores - scores.amax(-1, keepdim=True))
    scores = scores / scores.sum(-1, keepdim=True)
    o = (scores.view(b, hk, -1, len(j)) @ gather(v, vs).contiguous()).view(b, h, len(t), -1).permute(0, 2, 1, 3)
    return o[t < new[:, None]].half()


def _plain_verify(s):
    p, q, x, u = s["p"], s["q"], s["drafted"].long(), s["u"]
    b, k = x.shape
    i = torch.arange(k, device="cuda")
    count = torch.full((b,), k, device="cuda") if s["count"] is None else s["count"].long()
    px = p[:, :k].gather(2, x[..., None])[..., 0]
    qx = torch.ones_like(px) if q is None else q.gather(2, x[..., None])[..., 0]
    n = torch.cumprod(((u[:, :k] * qx < px) & (i < count[:, None])).int(), 1).sum(1)
    rows = torch.arange(b, device="cuda")
    # the next token is a whole number, decided by where a running sum passes a bound: in 64 bits, as any order of additions then decides alike
    w = p[rows, n].double()
    at = torch.minimum(n, torch.full_like(n, k - 1))
    if q is None:
        less = torch.zeros_like(w).scatter_(1, x[rows, at][:, None], float("inf"))
    else:
        less = q[rows, at].double()
    rest = torch.where((n < count)[:, None], torch.clamp(w - less, min=0), w)
    w = torch.where((rest.sum(1) > 0)[:, None], rest, w)                           # (nothing is left where both say the same)
    c = torch.cumsum(w, 1)
    token = (c <= u[:, k:].double() * c[:, -1:]).sum(1)
    last = w.shape[1] - 1 - torch.flip(w > 0, [1]).int().argmax(1)
    token = torch.minimum(token, last).int()
    j = torch.arange(k + 1, device="cuda")
    drafted = torch.cat([s["drafted"], s["drafted"][:, :1]], 1)
    tokens = torch.where(j < n[:, None], drafted, torch.where(j == n[:, None], token[:, None], torch.full_like(drafted, -1)))
    return tokens, n.int()


def run(state):
    kind = state["kind"]
    if own:
        return {"product": _own_product, "cache": _own_cache, "attention": _own_attention, "verify": _own_verify}[kind](state)
    return {"product": _plain_product, "cache": _plain_cache, "attention": _plain_attention, "verify": _plain_verify}[kind](state)


# ---- what a pass cannot do without, and what it returns in 64 bits --------------------------------------------------------------------

def _row_bytes(dim, bits):
    return dim * bits / 8 + (0 if bits == 16 else 4)


def work(case):
    if case["kind"] == "product":
        m, n, nb, value = case["m"], case["n"], case["nb"], 4 if case["fp32"] else 2
        entries = case["density"] * m * n
        y = m * nb * value
        return {"bytes": entries * (value + case["bits"] / 8) + n * nb * value + y * (1 + case["gate"] + case["residual"]) + case["bias"] * m * value,
                "flops": 2.0 * entries * nb}
    if case["kind"] == "cache":
        rows = 2 * case["tokens"] * case["heads"]
        # the new values once, the cached ones written and read, the values read back written
        return {"bytes": rows * (4 * case["dim"] + 2 * _row_bytes(case["dim"], case["bits"])) + 8 * case["tokens"], "flops": 4.0 * rows * case["dim"]}
    if case["kind"] == "attention":
        new, total = _lengths(case)
        pairs = sum(n * (t - n) + n * (n + 1) / 2 for n, t in zip(new, total))
        return {"bytes": 2 * sum(total) * case["kv_heads"] * _row_bytes(case["dim"], case["bits"]) + 4 * sum(new) * case["heads"] * case["dim"],
                "flops": 4.0 * pairs * case["heads"] * case["dim"]}
    rows = 1 if case["greedy"] else 2
    return {"bytes": case["batch"] * (4.0 * case["vocab"] * rows + 20 * case["drafts"]), "flops": 3.0 * case["batch"] * case["vocab"]}


def _exact_values(x, bits):
    """What the cache stands for, in 64 bits, from the definition of its steps."""
    x = x.double()
    if bits == 16:
        return x
    if bits == 8:
        step = x.abs().max(dim=-1, keepdim=True).values / 127
        return torch.where(step > 0, torch.round(x / step.clamp(min=1e-300)), 0.0) * step
    low = x.min(dim=-1, keepdim=True).values
    step = ((x.max(dim=-1, keepdim=True).values - low) / 15).half().double()
    return low + step * torch.where(step > 0, torch.round((x - low) / step.clamp(min=1e-300)).clamp(0, 15), 0.0)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "product":
        y = torch.cat([w.double() @ s["x"].double() for w in s["w"].split(2048)])
        if case["bias"]:
            y = (y.t() + s["bias"].double()).t()
        y = {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v),
             "gelu": lambda v: v * 0.5 * torch.erfc(-v * math.sqrt(0.5))}[case["act"]](y)
        if case["gate"]:
            y = y * s["gate"].double()
        return y + s["residual"].double() if case["residual"] else y
    if case["kind"] == "cache":
        return [_exact_values(s["k"], case["bits"]), _exact_values(s["v"], case["bits"])]
    if case["kind"] == "verify":
        return None                                          # whole numbers: they have to be equal
    new, total = _lengths(case)
    group, out, at = case["heads"] // case["kv_heads"], [], 0
    k, ks, v, vs = s["cache"]
    for i in range(case["batch"]):
        where = s["table"][i, :-(-total[i] // case["page"])].long()

        def sequence(code, step):
            x = _decode(code[where], None if step is None else step[where], case["bits"], torch.float64)
            return x.transpose(1, 2).reshape(-1, case["kv_heads"], case["dim"])[:total[i]]
        kk, vv = sequence(k, ks), sequence(v, vs)
        q = s["q"][at:at + new[i]].double()
        hidden = torch.arange(total[i], device="cuda") > torch.arange(total[i] - new[i], total[i], device="cuda")[:, None]
        o = torch.empty((new[i], case["heads"], case["dim"]), dtype=torch.float64, device="cuda")
        for h in range(case["heads"]):
            a = (q[:, h].contiguous() @ kk[:, h // group].t().contiguous()) / math.sqrt(case["dim"])
            o[:, h] = torch.softmax(a.masked_fill_(hidden, -math.inf), -1) @ vv[:, h // group].contiguous()
        out.append(o)
        at += new[i]
    return torch.cat(out)
