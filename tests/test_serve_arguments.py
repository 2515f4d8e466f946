"""What the calls around the products refuse, and what they launch, on a stand-in for the runtime."""
import standin

CODE = r"""
import ctypes
def cache(**o):
    d = dict(bits=8, pages=4, heads=2, page_size=16, head_dim=64, k=0x100000, v=0x200000, k_step=0x300000, v_step=0x400000)
    d.update(o)
    return B.KvCacheDesc(ctypes.sizeof(B.KvCacheDesc), **d)
def view(data=0x500000, t=128, h=64, d=1):
    return B.View(data, t, h, d)
def attention(**o):
    d = dict(q_heads=4, tokens=3, batch=2, max_pages=4, max_new=2, scale=0.125, table_stride=4, q_start=0x600000, kv_len=0x600100,
             page_table=0x600200, q=view(0x700000, 256), out=view(0x710000, 256))
    d.update(o)
    return B.AttentionDesc(ctypes.sizeof(B.AttentionDesc), **d)
def verify(**o):
    d = dict(batch=2, drafts=3, vocab=100, target=0x100000, draft=0x200000, uniform=0x300000, target_seq=400, target_row=100, draft_seq=300,
             draft_row=100, drafted=0x400000, count=0x500000, tokens=0x600000, accepted=0x700000)
    d.update(o)
    return B.VerifyDesc(ctypes.sizeof(B.VerifyDesc), **d)
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
    out[name] = [outcome(lambda: B.ecspmv_kv_write(cache(**cs), view(), view(), 0x800000, 5, stream[0])),
                 outcome(lambda: B.ecspmv_kv_read(cache(**cs), 0x800000, 5, view(), view(), stream[0])),
                 outcome(lambda: B.ecspmv_attention(cache(**cs), attention(), 0x900000, 1 << 30, stream[0])),
                 outcome(lambda: B.ecspmv_attention_workspace(cache(**cs), attention()))]
for name, o in arg["rows"]:
    o = dict(dict(k=0x500000, v=0x500000, slots=0x800000, tokens=5), **o)
    out[name] = [outcome(lambda: B.ecspmv_kv_write(cache(), view(o["k"]), view(o["v"]), o["slots"], o["tokens"], stream[0])),
                 outcome(lambda: B.ecspmv_kv_read(cache(), o["slots"], o["tokens"], view(o["k"]), view(o["v"]), stream[0]))]
for name, o in arg["attention"]:
    work, size = o.pop("work", 0x900000), o.pop("size", 1 << 30)
    for key in ("q", "out"):
        if key in o:
            o[key] = view(o[key], 256)
    out[name] = outcome(lambda: B.ecspmv_attention(cache(), attention(**o), work, size, stream[0]))
for name, o in arg["verify"]:
    out[name] = outcome(lambda: B.ecspmv_verify(verify(**o), 0x900000, 1 << 20, stream[0]))
A = B.ecspmv_build_dense(np.ones((16, 128), np.float16), B.make_opts())
F = B.ecspmv_build_dense_f32(np.ones((16, 128), np.float32), B.make_opts())
early = outcome(lambda: A.ecspmv_run_epilogue(0x100000, 0x200000, 1, B.Epilogue(ctypes.sizeof(B.Epilogue), 1, 0, 0, 0), stream[0]))
for M in (A, F):
    M.ecspmv_upload(0x100000, M.ecspmv_device_bytes(), 0)
out["early"] = early
for name, f32, nb, fields in arg["epilogue"]:
    e = B.Epilogue(ctypes.sizeof(B.Epilogue), *fields)
    out[name] = outcome(lambda: (F if f32 else A).ecspmv_run_epilogue(0x100000, 0x200000, nb, e, stream[0]))
L = B.lib()
out["no epilogue"] = [L.ecspmv_run_epilogue(A._h, 0x100000, 0x200000, 1, None, 0), L.ecspmv_run_epilogue(None, 0x100000, 0x200000, 1, B.Epilogue(32), 0)]
short = cache()
short.struct_size = 3
out["short"] = [L.ecspmv_kv_write(short, view(), view(), 0x800000, 5, 0), L.ecspmv_kv_write(None, view(), view(), 0x800000, 5, 0),
                L.ecspmv_kv_write(cache(), None, view(), 0x800000, 5, 0), L.ecspmv_attention(cache(), None, 0, 0, 0),
                L.ecspmv_attention_workspace(cache(), attention(), None), L.ecspmv_verify(None, 0x900000, 1 << 20, 0)]
long = attention(max_pages=100, table_stride=100)
out["work"] = B.ecspmv_attention_workspace(cache(), long)
out["enough"] = [outcome(lambda: B.ecspmv_attention(cache(), long, 0x900000, out["work"] - d, stream[0])) for d in (0, 1)]
out["grid"] = fake.fake_launched(GRID)
out["none"] = outcome(lambda: B.ecspmv_attention(cache(), long, 0, out["work"], stream[0]))
need = B.ecspmv_verify_workspace(verify())
out["verify work"] = [need, outcome(lambda: B.ecspmv_verify(verify(), 0x900000, need, stream[0])),
                      outcome(lambda: B.ecspmv_verify(verify(), 0x900000, need - 1, stream[0])),
                      outcome(lambda: B.ecspmv_verify(verify(), 0x900004, need, stream[0])), outcome(lambda: B.ecspmv_verify(verify(), 0, need, stream[0]))]
out["stream"] = []
for s in (0x1000, 0x2000, 0):
    B.ecspmv_verify(verify(), 0x900000, 1 << 20, s)
    out["stream"].append([fake.fake_launched(STREAM), fake.fake_launched(KERNEL)])
try:
    B.ecspmv_verify(verify(), 0x900000, 1 << 20, 0x3000)
except B.EcspmvError as e:
    out["stream"].append(e.status)
print(json.dumps(out))
"""

CACHE = [("ok", {}), ("16 bits", dict(bits=16, k_step=0, v_step=0)), ("bits", dict(bits=5)), ("no k", dict(k=0)), ("k off", dict(k=0x100008)),
         ("no step", dict(k_step=0)), ("step off", dict(v_step=0x400004)), ("page 8", dict(page_size=8)), ("page 48", dict(page_size=48)),
         ("page 2048", dict(page_size=2048)), ("dim 8", dict(head_dim=8)), ("dim 72", dict(head_dim=72)), ("dim 272", dict(head_dim=272)),
         ("no pages", dict(pages=0)), ("no heads", dict(heads=0))]
ROWS = [("rows off", dict(k=0x500001)), ("no v", dict(v=0)), ("no slots", dict(slots=0)), ("slots off", dict(slots=0x800004)),
        ("tokens -1", dict(tokens=-1)), ("no tokens", dict(tokens=0, k=0, v=0, slots=0)), ("tokens", dict(tokens=1 << 31))]
ATTENTION = [("a ok", {}), ("group", dict(q_heads=3)), ("no q heads", dict(q_heads=0)), ("no out", dict(out=0)), ("q off", dict(q=0x700001)),
             ("no start", dict(q_start=0)), ("no len", dict(kv_len=0)), ("len off", dict(kv_len=0x600102)), ("no table", dict(page_table=0)),
             ("stride", dict(table_stride=3)), ("batch -1", dict(batch=-1)), ("nothing", dict(tokens=0, q=0, out=0)), ("no batch", dict(batch=0)),
             ("no new", dict(max_new=0)), ("batch", dict(batch=65536)), ("pages", dict(max_pages=1 << 30, table_stride=1 << 30)),
             ("no keys", dict(max_pages=0, page_table=0, table_stride=0))]
VERIFY = [("v ok", {}), ("v plain", dict(draft=0, count=0)), ("no vocab", dict(vocab=0)), ("vocab", dict(vocab=(1 << 20) + 1)), ("drafts -1", dict(drafts=-1)),
          ("no drafts", dict(drafts=0, drafted=0, draft=0)), ("no drafted", dict(drafted=0)), ("no target", dict(target=0)),
          ("target off", dict(target=0x100002)), ("no sequences", dict(batch=0, target=0)), ("no uniform", dict(uniform=0)),
          ("no accepted", dict(accepted=0))]
EPILOGUE = [("e ok", 0, 1, [2, 0x300000, 0x300002, 0x300004]), ("e none", 0, 1, [0, 0, 0, 0]), ("e multi", 0, 4, [1, 0, 0, 0x300000]),
            ("e f32", 1, 8, [3, 0x300004, 0, 0]), ("e act", 0, 1, [4, 0, 0, 0]), ("e act -1", 0, 1, [-1, 0, 0, 0]), ("e nb", 0, 3, [1, 0, 0, 0]),
            ("e off", 0, 1, [0, 0x300001, 0, 0]), ("e f32 off", 1, 1, [0, 0, 0x300002, 0]), ("e f32 off residual", 1, 2, [0, 0, 0, 0x300002])]
INVALID, UNSUPPORTED, HIP, SMALL = -1, -2, -4, -6


def test_refusals(tmp_path):
    got = standin.run(tmp_path, CODE, dict(cache=CACHE, rows=ROWS, attention=ATTENTION, verify=VERIFY, epilogue=EPILOGUE))
    for name, _ in CACHE:
        want = {"bits": UNSUPPORTED, "page 8": UNSUPPORTED, "page 48": UNSUPPORTED, "page 2048": UNSUPPORTED, "dim 8": UNSUPPORTED,
                "dim 72": UNSUPPORTED, "dim 272": UNSUPPORTED, "ok": 0, "16 bits": 0}.get(name, INVALID)
        assert got[name] == ([1, 1, 1, 0] if want == 0 else [[want, 0]] * 4), (name, got[name])
    for name, _ in ROWS:
        want = {"no tokens": 0, "tokens": [UNSUPPORTED, 0]}.get(name, [INVALID, 0])
        assert got[name] == [want, want], (name, got[name])
    for name, _ in ATTENTION:
        want = {"a ok": 1, "no keys": 1, "nothing": 0, "no batch": 0, "no new": 0, "batch": [UNSUPPORTED, 0], "pages": [UNSUPPORTED, 0]}.get(
            name, [INVALID, 0])
        assert got[name] == want, (name, got[name])
    for name, _ in VERIFY:
        want = {"v ok": 1, "v plain": 1, "no drafts": 1, "no sequences": 0, "vocab": [UNSUPPORTED, 0]}.get(name, [INVALID, 0])
        assert got[name] == want, (name, got[name])
    for name, *_ in EPILOGUE:
        want = {"e ok": 1, "e none": 1, "e multi": 1, "e f32": 1, "e act": [UNSUPPORTED, 0], "e act -1": [UNSUPPORTED, 0]}.get(name, [INVALID, 0])
        assert got[name] == want, (name, got[name])
    assert got["early"] == [-5, 0] and got["no epilogue"] == [INVALID, INVALID]
    assert got["short"] == [INVALID] * 6
    assert got["work"] > 0 and got["enough"] == [1, [SMALL, 0]] and got["grid"] == 3 * 4 and got["none"] == [INVALID, 0]
    assert got["verify work"] == [2 * 2 * 8, 1, [SMALL, 0], [INVALID, 0], [INVALID, 0]]
    assert got["stream"] == [[0x1000, 0x100], [0x2000, 0x200], [0, 0x100], HIP]
