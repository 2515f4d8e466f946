"""What the calls of decoding with trees refuse, and what they launch, on a stand-in for the runtime."""
import standin

CODE = r"""
import ctypes
def cache(**o):
    d = dict(bits=8, pages=4, heads=2, page_size=16, head_dim=64, k=0x100000, v=0x200000, k_step=0x300000, v_step=0x400000)
    d.update(o)
    return B.KvCacheDesc(ctypes.sizeof(B.KvCacheDesc), **d)
def view(data=0x500000, t=128, h=64, d=1):
    return B.View(data, t, h, d)
def rotary(**o):
    d = dict(rotary_dim=64, neighbours=0, q_heads=4, frequency=0xA00000, position=0xB00000, q=0x700000, q_out=0x710000)
    for name in ("q", "q_out"):
        d.update({name + "_token_stride": 256, name + "_head_stride": 64, name + "_dim_stride": 1})
    d.update(o)
    return B.RotaryDesc(ctypes.sizeof(B.RotaryDesc), **d)
def attention(**o):
    d = dict(q_heads=4, tokens=3, batch=2, max_pages=4, max_new=2, scale=0.125, table_stride=4, q_start=0x600000, kv_len=0x600100,
             page_table=0x600200, q=view(0x700000, 256), out=view(0x710000, 256))
    d.update(o)
    return B.AttentionDesc(ctypes.sizeof(B.AttentionDesc), **d)
def keep(**o):
    d = dict(batch=2, nodes=5, max_pages=4, path_stride=5, table_stride=4, first=0x100000, path=0x200000, accepted=0x300000, page_table=0x400000)
    d.update(o)
    return B.KeepDesc(ctypes.sizeof(B.KeepDesc), **d)
def verify(**o):
    d = dict(batch=2, nodes=3, vocab=100, target=0x100000, uniform=0x300000, target_seq=400, target_row=100, drafted=0x400000, parent=0x480000,
             count=0x500000, tokens=0x600000, path=0x680000, accepted=0x700000)
    d.update(o)
    return B.VerifyTreeDesc(ctypes.sizeof(B.VerifyTreeDesc), **d)
stream = [0x1000]
def outcome(f):
    # whether something was launched (streams 0x1000 ... 0x1fff are the first device's), or the status
    stream[0] += 1
    try:
        f()
        status = 0
    except B.EcspmvError as e:
        status = e.status
    launched = int(fake.fake_launched(STREAM) == stream[0])
    return [status, launched] if status else launched
out = {}
for name, cs in arg["cache"]:
    out[name] = [outcome(lambda: B.ecspmv_kv_append(cache(**cs), view(), view(), 0x800000, 5, rotary(rotary_dim=16), stream[0])),
                 outcome(lambda: B.ecspmv_attention_tree(cache(**cs), attention(), 0xC00000, 1, 0x900000, 1 << 30, stream[0])),
                 outcome(lambda: B.ecspmv_kv_keep(B.cache_array([cache(**cs)] * 2), keep(), stream[0]))]
for name, o in arg["append"]:
    at = {k: o.pop(k) for k in ("k", "v", "slots", "tokens") if k in o}
    out[name] = outcome(lambda: B.ecspmv_kv_append(cache(), view(at.get("k", 0x500000)), view(at.get("v", 0x500000)), at.get("slots", 0x800000),
                                                   at.get("tokens", 5), rotary(**o), stream[0]))
for name, o in arg["attention"]:
    work, size, seen, stride = (o.pop(k, d) for k, d in (("work", 0x900000), ("size", 1 << 30), ("seen", 0xC00000), ("stride", 1)))
    out[name] = outcome(lambda: B.ecspmv_attention_tree(cache(), attention(**o), seen, stride, work, size, stream[0]))
for name, o in arg["keep"]:
    count = o.pop("count", 2)
    out[name] = outcome(lambda: B.ecspmv_kv_keep(B.cache_array([cache()] * count), keep(**o), stream[0]))
for name, o in arg["verify"]:
    out[name] = outcome(lambda: B.ecspmv_verify_tree(verify(**o), 0x900000, 1 << 20, stream[0]))
for name, strides in arg["out"]:
    out[name] = outcome(lambda: B.ecspmv_attention_tree(cache(), attention(out=view(0x710000, *strides)), 0xC00000, 1, 0x900000, 1 << 30, stream[0]))
out["unlike"] = [outcome(lambda: B.ecspmv_kv_keep(B.cache_array([cache(), cache(**o)]), keep(), stream[0]))
                 for o in (dict(pages=5), dict(heads=3), dict(page_size=32), dict(head_dim=48), dict(bits=4), dict(k=0x900000))]
# a later cache that is refused: nothing is launched for the ones before it
out["late"] = outcome(lambda: B.ecspmv_kv_keep(B.cache_array([cache()] * 70 + [cache(v=0)]), keep(), stream[0]))
B.ecspmv_kv_keep(B.cache_array([cache()] * 70), keep(), 0x1000)
out["layers"] = fake.fake_launched(GRID)
L = B.lib()
short = rotary()
short.struct_size = 3
out["short"] = [L.ecspmv_kv_append(cache(), view(), view(), 0x800000, 5, short, 0), L.ecspmv_kv_append(cache(), view(), view(), 0x800000, 5, None, 0),
                L.ecspmv_kv_append(None, view(), view(), 0x800000, 5, rotary(), 0), L.ecspmv_kv_append(cache(), None, view(), 0x800000, 5, rotary(), 0),
                L.ecspmv_kv_keep(None, 1, keep(), 0), L.ecspmv_kv_keep(B.cache_array([cache()]), 1, None, 0),
                L.ecspmv_kv_keep(B.cache_array([cache()]), -1, keep(), 0),
                L.ecspmv_kv_keep((ctypes.POINTER(B.KvCacheDesc) * 1)(), 1, keep(), 0),
                L.ecspmv_attention_tree(cache(), None, 0xC00000, 1, 0, 0, 0), L.ecspmv_verify_tree(None, 0x900000, 1 << 20, 0),
                L.ecspmv_verify_tree_workspace(verify(), None)]
long = attention(max_pages=100, table_stride=100)
work = B.ecspmv_attention_tree_workspace(cache(), long)
out["enough"] = [outcome(lambda: B.ecspmv_attention_tree(cache(), long, 0xC00000, 1, 0x900000, work - d, stream[0])) for d in (0, 1)]
out["none"] = outcome(lambda: B.ecspmv_attention_tree(cache(), long, 0xC00000, 1, 0, work, stream[0]))
need = B.ecspmv_verify_tree_workspace(verify())
out["verify work"] = [need, outcome(lambda: B.ecspmv_verify_tree(verify(), 0x900000, need, stream[0])),
                      outcome(lambda: B.ecspmv_verify_tree(verify(), 0x900000, need - 1, stream[0])),
                      outcome(lambda: B.ecspmv_verify_tree(verify(), 0x900004, need, stream[0])),
                      outcome(lambda: B.ecspmv_verify_tree(verify(), 0, need, stream[0]))]
calls = [lambda s: B.ecspmv_kv_append(cache(), view(), view(), 0x800000, 5, rotary(), s),
         lambda s: B.ecspmv_attention_tree(cache(), attention(), 0xC00000, 1, 0x900000, 1 << 30, s),
         lambda s: B.ecspmv_kv_keep(B.cache_array([cache()]), keep(), s),
         lambda s: B.ecspmv_verify_tree(verify(), 0x900000, 1 << 20, s)]
out["stream"] = []
for call in calls:
    for s in (0x1000, 0x2000, 0):
        call(s)
        out["stream"].append([fake.fake_launched(STREAM), fake.fake_launched(KERNEL)])
    try:
        call(0x3000)
    except B.EcspmvError as e:
        out["stream"].append(e.status)
# the longest runs of tokens and the most heads: a grid that a launch takes
out["grid"] = []
for tokens, q_heads in ((1 << 27, 1), (1, 65535), (100000, 1000)):
    B.ecspmv_kv_append(cache(), view(), view(), 0x800000, tokens, rotary(q_heads=q_heads), 0x1000)
    out["grid"].append(fake.fake_launched(GRID) * 256)
print(json.dumps(out))
"""

CACHE = [("ok", {}), ("16 bits", dict(bits=16, k_step=0, v_step=0)), ("bits", dict(bits=5)), ("no k", dict(k=0)), ("v off", dict(v=0x100008)),
         ("no step", dict(k_step=0)), ("step off", dict(v_step=0x400004)), ("page 48", dict(page_size=48)), ("dim 72", dict(head_dim=72)),
         ("no pages", dict(pages=0)), ("no heads", dict(heads=0))]
APPEND = [("p ok", {}), ("p none", dict(rotary_dim=0, frequency=0, position=0)), ("p no q", dict(q_heads=0, q=0, q_out=0)), ("p odd", dict(rotary_dim=63)),
          ("p wide", dict(rotary_dim=66)), ("p below", dict(rotary_dim=-2)), ("p heads -1", dict(q_heads=-1)), ("p pairs", dict(neighbours=2)),
          ("p no frequency", dict(frequency=0)), ("p frequency off", dict(frequency=0xA00004)), ("p no position", dict(position=0)),
          ("p position off", dict(position=0xB00002)), ("p no q_out", dict(q_out=0)), ("p q off", dict(q=0x700001)), ("p no k", dict(k=0)),
          ("p no slots", dict(slots=0)), ("p slots off", dict(slots=0x800004)), ("p tokens -1", dict(tokens=-1)),
          ("p nothing", dict(tokens=0, k=0, v=0, slots=0, q=0)), ("p tokens", dict(tokens=(1 << 27) + 1)), ("p rows", dict(tokens=1 << 20, q_heads=2048)),
          ("p q heads", dict(q_heads=65536)),
          ("p q_out of a token", dict(q_out_token_stride=0)), ("p q_out of a head", dict(q_out_head_stride=0)), ("p q_out of a value", dict(q_out_dim_stride=0)),
          ("p one token", dict(tokens=1, q_out_token_stride=0)), ("p q of a token", dict(q_token_stride=0))]
ATTENTION = [("a ok", {}), ("no seen", dict(seen=0)), ("seen off", dict(seen=0xC00002)), ("seen stride", dict(stride=0)),
             ("words", dict(tokens=100, max_new=65, stride=2)), ("words enough", dict(tokens=100, max_new=65, stride=3)),
             ("words of tokens", dict(tokens=32, max_new=1000, stride=1)), ("group", dict(q_heads=3)), ("no start", dict(q_start=0)),
             ("no table", dict(page_table=0)), ("nothing", dict(tokens=0)), ("no batch", dict(batch=0, seen=0)), ("no new", dict(max_new=0))]
OUT = [("o token", (0, 64, 1)), ("o head", (256, 0, 1)), ("o value", (256, 64, 0)), ("o ok", (-256, 64, 1))]
KEEP = [("k ok", {}), ("k nothing", dict(nodes=0, path=0, path_stride=0)), ("k no batch", dict(batch=0)), ("k no caches", dict(count=0)),
        ("k no pages", dict(max_pages=0, page_table=0)), ("k batch -1", dict(batch=-1)), ("k batch", dict(batch=65536)), ("k nodes -1", dict(nodes=-1)),
        ("k pages -1", dict(max_pages=-1)), ("k path stride", dict(path_stride=4)), ("k table stride", dict(table_stride=3)), ("k no path", dict(path=0)),
        ("k no first", dict(first=0)), ("k accepted off", dict(accepted=0x300002)), ("k no table", dict(page_table=0)),
        ("k pages", dict(max_pages=1 << 30, table_stride=1 << 30))]
VERIFY = [("v ok", {}), ("v all", dict(count=0)), ("no vocab", dict(vocab=0)), ("vocab", dict(vocab=(1 << 20) + 1)), ("nodes -1", dict(nodes=-1)),
          ("nodes", dict(nodes=1025)), ("no nodes", dict(nodes=0, drafted=0, parent=0, path=0)), ("no drafted", dict(drafted=0)),
          ("no parent", dict(parent=0)), ("no path", dict(path=0)), ("no target", dict(target=0)), ("parent off", dict(parent=0x480002)),
          ("no sequences", dict(batch=0, target=0)), ("no uniform", dict(uniform=0)), ("no tokens", dict(tokens=0)), ("v batch", dict(batch=65536))]
INVALID, UNSUPPORTED, HIP, SMALL = -1, -2, -4, -6


def test_refusals(tmp_path):
    got = standin.run(tmp_path, CODE, dict(cache=CACHE, append=APPEND, attention=ATTENTION, keep=KEEP, verify=VERIFY, out=OUT))

    def holds(cases, right, unsupported=()):
        for name, _ in cases:
            want = right.get(name, [UNSUPPORTED if name in unsupported else INVALID, 0])
            assert got[name] == want, (name, got[name])
    holds(CACHE, {"ok": [1] * 3, "16 bits": [1] * 3, **{n: [[UNSUPPORTED, 0]] * 3 for n in ("bits", "page 48", "dim 72")},
                  **{n: [[INVALID, 0]] * 3 for n in ("no k", "v off", "no step", "step off", "no pages", "no heads")}})
    holds(APPEND, {"p ok": 1, "p none": 1, "p no q": 1, "p nothing": 0, "p one token": 1, "p q of a token": 1}, ("p pairs", "p tokens", "p rows", "p q heads"))
    holds(ATTENTION, {"a ok": 1, "words enough": 1, "words of tokens": 1, "nothing": 0, "no batch": 0, "no new": 0})
    holds(OUT, {"o ok": 1})
    holds(KEEP, {"k ok": 1, "k nothing": 0, "k no batch": 0, "k no caches": 0, "k no pages": 0}, ("k batch", "k pages"))
    holds(VERIFY, {"v ok": 1, "v all": 1, "no nodes": 1, "no sequences": 0}, ("vocab", "nodes", "v batch"))
    assert got["unlike"] == [[INVALID, 0]] * 5 + [1] and got["late"] == [INVALID, 0]
    assert got["layers"] == 2 * 6                            # 64 caches in the first launch, 6 in the second
    assert got["short"] == [INVALID] * 11
    assert got["enough"] == [1, [SMALL, 0]] and got["none"] == [INVALID, 0]
    assert got["verify work"] == [2 * (8 + 16 + 16), 1, [SMALL, 0], [INVALID, 0], [INVALID, 0]]
    assert got["stream"] == [[0x1000, 0x100], [0x2000, 0x200], [0, 0x100], HIP] * 4
    assert all(g < 1 << 32 for g in got["grid"])


OVERLAP = r"""
import ctypes
c = B.KvCacheDesc(ctypes.sizeof(B.KvCacheDesc), bits=16, pages=4, heads=2, page_size=16, head_dim=64, k=0x100000, v=0x200000)
def append(q, q_out, q_heads=2):
    r = B.RotaryDesc(ctypes.sizeof(B.RotaryDesc), rotary_dim=64, neighbours=0, q_heads=q_heads, frequency=0xA00000, position=0xB00000, q=q, q_out=q_out)
    for name in ("q", "q_out"):
        for what, stride in (("token", 128), ("head", 64), ("dim", 1)):
            setattr(r, f"{name}_{what}_stride", stride)
    try:
        B.ecspmv_kv_append(c, B.View(0x500000, 128, 64, 1), B.View(0x600000, 128, 64, 1), 0x800000, 5, r, 0x1000)
    except B.EcspmvError as e:
        return e.status
    return 0
print(json.dumps([append(*a) for a in arg]))
"""


def test_queries_do_not_go_where_keys_or_values_are_read(tmp_path):
    """q_out is written while others still read k and v; q may lie there, q_out may be q, and without queries it is not looked at."""
    k, v, q, out = 0x500000, 0x600000, 0x700000, 0x710000
    calls = [(q, out), (q, q), (k, out), (v, out), (q, k), (q, v), (k, k), (v, v), (q, k, 0)]
    assert standin.run(tmp_path, OVERLAP, calls) == [0, 0, 0, 0, INVALID, INVALID, INVALID, INVALID, 0]
