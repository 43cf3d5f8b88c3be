"""What the calls on clear activations refuse, without a GPU: every wrong argument is answered with its code and a message before anything is
launched, and good ones launch on the stream that they are given."""
import pytest

from simhip import run

PROGRAM = """
import struct
ctx = binding.Context(12, 36, 3, 37, 1, 1, 30)
lib = ctx.lib
BADARG, SHAPE = -1, -4
where = [1 << 20]
def at(n):  # an address of its own for n bytes (nothing is read: kernels do not run)
    where[0] += (n + 4095) // 4096 * 4096 + 4096
    return where[0]
def refused(rc, code, text=""):
    message = lib.ensi_last_error(ctx.h).decode()
    assert rc == code and text in message, (rc, code, message)
st = 4096
"""


def launches(calls):
    return [c for c in calls if c[0] == "launch" and "k_clear_" in c[2]]


def names(calls):
    return [c[2] for c in launches(calls)]


def test_null_arguments(tmp_path):
    run(tmp_path, PROGRAM + """
n = None
assert lib.ensi_clear_norm(n, b"", n) == -1 and lib.ensi_clear_norm(ctx.h, n, n) == -1
assert lib.ensi_clear_weights_prepare(n, n, n, 1, 1, 0, n) == -1
assert lib.ensi_clear_matmul(n, n, n, 0, n, n, 0, 1, 0, n) == -1 and lib.ensi_clear_matmul(ctx.h, n, n, 0, n, n, 0, 1, 0, n) == -1
assert lib.ensi_clear_cache_wrap(n, n, n, n, n, 1, 1, 16, 64, n) == -1
assert lib.ensi_clear_cache_status(n, n, n, n) == -1
assert lib.ensi_clear_append(n, n, b"", n) == -1 and lib.ensi_clear_append(ctx.h, n, b"", n) == -1
assert lib.ensi_clear_attention(n, n, b"", n) == -1 and lib.ensi_clear_attention(ctx.h, n, b"", n) == -1
lib.ensi_clear_weights_free(n)
lib.ensi_clear_cache_free(n)
""")


def test_norm(tmp_path):
    calls = run(tmp_path, PROGRAM + """
def norm(code=None, text="", **over):
    a = dict(x=at(4096), residual=0, gain=at(4096), sum_out=0, out=0, codes=at(4096), scales=at(4096), rows=4, x_stride=64, residual_stride=0, sum_stride=0, out_stride=0,
             d=64, type=1, eps=1e-5)
    a.update(over)
    rc = lib.ensi_clear_norm(ctx.h, binding._NORM.pack(*a.values(), 0), st)
    if code is None:
        assert rc == 0, lib.ensi_last_error(ctx.h)
    else:
        refused(rc, code, text)
mark("good")
norm()
norm(rows=0, x=0, gain=0)
x, r = at(4096), at(4096)
norm(x=x, residual=r, residual_stride=64, sum_out=r, sum_stride=64)
norm(x=x, residual=r, residual_stride=64, sum_out=x, sum_stride=64)
norm(x=x, out=x, out_stride=64)
norm(x_stride=70, d=64)
mark("bad")
norm(BADARG, "type", type=3)
norm(SHAPE, "elements", d=0)
norm(SHAPE, "elements", d=32769)
norm(SHAPE, "elements", rows=-1)
norm(SHAPE, "elements", rows=(1 << 21) + 1)
norm(BADARG, "eps", eps=-1.0)
norm(BADARG, "eps", eps=float("nan"))
norm(BADARG, "gain", gain=0)
norm(BADARG, "wanted", codes=0, scales=0)
norm(BADARG, "together", scales=0)
norm(BADARG, "residual", sum_out=at(4096), sum_stride=64)
norm(SHAPE, "overlap", x_stride=63)
norm(BADARG, "overlaps", x=x, out=x + 128, out_stride=64)
norm(BADARG, "overlaps", x=x, out=x, out_stride=65, x_stride=64)
norm(BADARG, "overlaps", x=x, codes=x)
norm(BADARG, "overlaps", x=x, residual=r, residual_stride=64, sum_out=x, sum_stride=65)
g = at(4096)
norm(BADARG, "overlaps", gain=g, scales=g + 64)
""")
    assert len(launches(calls)) == 5 and all(c[1] == "0x1000" for c in launches(calls))


def test_weights_and_matmul(tmp_path):
    calls = run(tmp_path, PROGRAM + """
import ctypes
W, s = np.zeros((100, 30), dtype=np.int8), np.ones((2, 30), dtype=np.float32)
cw = ctypes.c_void_p()
prepare = lambda d, m, group: lib.ensi_clear_weights_prepare(ctx.h, binding._ptr(W), binding._ptr(s), d, m, group, ctypes.byref(cw))
refused(prepare(0, 30, 0), SHAPE, "131072")
refused(prepare(131073, 1, 0), SHAPE, "131072")
refused(prepare(100, 0, 0), SHAPE, "2^24")
refused(prepare(100, 30, 32), SHAPE, "multiple of 64")
refused(prepare(100, 30, -64), SHAPE, "multiple of 64")
for bad in (lambda: ctx.clear_weights_prepare(W.astype(np.int32), s, 64), lambda: ctx.clear_weights_prepare(W[0], s, 64), lambda: ctx.clear_weights_prepare(W, s, 0),
            lambda: ctx.clear_weights_prepare(W, s.T.copy(), 64), lambda: ctx.clear_weights_prepare(W, s, 48)):
    try:
        bad()
    except binding.EnsiError:
        continue
    raise AssertionError("not refused")
mark("good")
w = ctx.clear_weights_prepare(W, s, 64)
codes, scales, out = at(1 << 20), at(4096), at(1 << 20)
def mm(code=None, text="", codes=codes, stride=100, scales=scales, out=out, out_stride=30, rows=5, type=2):
    rc = lib.ensi_clear_matmul(ctx.h, w.h, codes, stride, scales, out, out_stride, rows, type, st)
    if code is None:
        assert rc == 0, lib.ensi_last_error(ctx.h)
    else:
        refused(rc, code, text)
mm()
mm(rows=0, codes=None)
mm(rows=1, stride=0, out_stride=0)
mark("bad")
mm(BADARG, "type", type=-1)
mm(SHAPE, "rows", rows=-1)
mm(SHAPE, "rows", rows=(1 << 20) + 1)
mm(BADARG, "null", codes=None)
mm(BADARG, "null", scales=None)
mm(SHAPE, "overlap", stride=99)
mm(SHAPE, "overlap", out_stride=29)
mm(BADARG, "overlaps", out=codes + 100)
mm(BADARG, "overlaps", out=scales)
other = binding.Context(12, 36, 3, 37, 1, 1, 30)
assert lib.ensi_clear_matmul(other.h, w.h, codes, 100, scales, out, 30, 5, 2, st) == -1
w.free()
""")
    assert [("pack" in n, "matmul" in n) for n in names(calls)] == [(True, False), (False, True), (False, True)]


CACHE = """
import ctypes
def wrap(pages=10, heads=2, page=32, dim=64, k=None, v=None, ks=None, vs=None):
    size = max(1, pages) * max(1, heads) * max(16, page) * max(1, dim)
    kv = ctypes.c_void_p()
    rc = lib.ensi_clear_cache_wrap(ctx.h, ctypes.c_void_p(k or at(size)), ctypes.c_void_p(v or at(size)), ctypes.c_void_p(ks or at(size)), ctypes.c_void_p(vs or at(size)), pages, heads, page, dim, ctypes.byref(kv))
    return rc, kv
"""


def test_cache(tmp_path):
    run(tmp_path, PROGRAM + CACHE + """
for bad in (dict(dim=32), dict(dim=100), dict(dim=512)):
    refused(wrap(**bad)[0], SHAPE, "heads of")
for bad in (dict(pages=0), dict(heads=0), dict(heads=4097), dict(page=8), dict(page=24)):
    refused(wrap(**bad)[0], SHAPE, "pages")
rc, kv = wrap(pages=1 << 30, heads=4096, page=16)
refused(rc, SHAPE, "2^31")
refused(wrap(k=(1 << 40) + 8)[0], BADARG, "aligned")
refused(wrap(ks=(1 << 40) + 2)[0], BADARG, "aligned")
k = at(1 << 20)
refused(wrap(k=k, v=k + 64)[0], BADARG, "overlap")
refused(wrap(k=k, vs=k)[0], BADARG, "overlap")
rc, kv = wrap()
assert rc == 0
bits = ctypes.c_int32(7)
assert lib.ensi_clear_cache_status(ctx.h, kv, ctypes.byref(bits), ctypes.c_void_p(st)) == 0 and bits.value == 0
other = binding.Context(12, 36, 3, 37, 1, 1, 30)
assert lib.ensi_clear_cache_status(other.h, kv, ctypes.byref(bits), None) == -1
lib.ensi_clear_cache_free(kv)
""")


def test_append_and_attention(tmp_path):
    calls = run(tmp_path, PROGRAM + CACHE + """
rc, kv = wrap()
assert rc == 0
def seqs(over):
    s = dict(begin=at(64), lengths=at(64), table=at(4096), table_stride=8, tokens=6, seqs=3, table_width=8, max_new=4)
    s.update({k: over.pop(k) for k in list(over) if k in s})
    return list(s.values()) + [0]
def check(rc, code, text):
    if code is None:
        assert rc == 0, lib.ensi_last_error(ctx.h)
    else:
        refused(rc, code, text)
def append(code=None, text="", **over):
    s = seqs(over)
    a = dict(q=at(1 << 16), k=at(1 << 16), v=at(1 << 16), q_out=at(1 << 16), cos=at(1 << 16), sin=at(1 << 16), q_stride=256, q_out_stride=256, k_stride=128, v_stride=128,
             q_heads=4, rot=64, positions=100, pairs=0, type=1)
    a.update(over)
    check(lib.ensi_clear_append(ctx.h, kv, binding._APPEND.pack(*s, *a.values(), 0), st), code, text)
def attention(code=None, text="", **over):
    s = seqs(over)
    a = dict(q=at(1 << 16), out=at(1 << 16), q_stride=256, out_stride=256, q_heads=4, type=1, score=0, window=0, max_length=200, cap=0.0, bias=0.0)
    a.update(over)
    check(lib.ensi_clear_attention(ctx.h, kv, binding._ATTENTION.pack(*s, *a.values(), 0), st), code, text)
mark("good")
append()
append(q=0, q_out=0, q_heads=0)
append(rot=0, cos=0, sin=0, positions=0)
q = at(1 << 16)
append(q=q, q_out=q)
qkv = at(1 << 16)  # one array of queries, keys and values: the rotated queries to their place
append(q=qkv, q_out=qkv, k=qkv + 512, v=qkv + 768, q_stride=512, q_out_stride=512, k_stride=512, v_stride=512)
append(tokens=0, k=0, v=0)
append(seqs=0, begin=0)
attention()
attention(max_new=1, max_length=100000)   # split: two launches
attention(seqs=0)
attention(max_length=0)
attention(score=1, window=5, cap=3.0, bias=-1.0)
mark("bad")
append(BADARG, "type", type=9)
append(BADARG, "pairs", pairs=2)
append(SHAPE, "multiple of 16", rot=24)
append(SHAPE, "multiple of 16", rot=80)
append(SHAPE, "multiple of 16", rot=-16)
append(SHAPE, "q_out", q_out=0)
append(SHAPE, "query heads", q_heads=0)
append(SHAPE, "positions", positions=-1)
append(BADARG, "null", k=0)
append(BADARG, "null", cos=0)
append(SHAPE, "overlap", k_stride=127)
append(SHAPE, "overlap", q_stride=255)
append(BADARG, "overlaps q", q=q, q_out=q + 512)
append(BADARG, "overlaps q", q=q, q_out=q, q_out_stride=300, q_stride=256)
append(BADARG, "k or v", k=q, q_out=q)
for f in (append, attention):
    f(SHAPE, "sequences", seqs=-1)
    f(SHAPE, "sequences", seqs=65536)
    f(SHAPE, "sequences", tokens=-1)
    f(SHAPE, "sequences", max_new=(1 << 20) + 1)
    f(BADARG, "table", table=0)
    f(BADARG, "table", begin=0)
    f(BADARG, "table", lengths=0)
    f(BADARG, "table", table_width=0)
    f(BADARG, "table", table_stride=7)
attention(BADARG, "type", type=0)
attention(BADARG, "score", score=2)
attention(SHAPE, "heads", q_heads=3)
attention(SHAPE, "heads", q_heads=0)
attention(SHAPE, "heads", q_heads=8192)
for bad in (dict(window=-1), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(bias=float("nan")), dict(max_length=-1), dict(max_length=(1 << 30) + 1)):
    attention(BADARG, "window", **bad)
attention(BADARG, "null", q=0)
attention(SHAPE, "overlap", q_stride=255)
attention(BADARG, "overlaps", q=q, out=q)
other = binding.Context(12, 36, 3, 37, 1, 1, 30)
assert lib.ensi_clear_append(other.h, kv, binding._APPEND.pack(*[0] * 25), st) == -1
lib.ensi_clear_cache_free(kv)
""")
    got = names(calls)
    assert sum("k_clear_append" in n for n in got) == 5 and sum("k_clear_attention_join" in n for n in got) >= 1 and all(c[1] == "0x1000" for c in launches(calls))
    marks = [i for i, c in enumerate(calls) if c[0] == "mark"]
    assert not launches(calls[marks[1]:])


def test_tensors_that_do_not_fit_are_refused_by_the_binding(tmp_path):
    """Shapes, types, devices and gaps are the binding's to check: on tensors of the host, which are on no device of the library."""
    pytest.importorskip("torch")
    run(tmp_path, PROGRAM + """
import torch
binding._TORCH = (lambda: -1, lambda at: 0, {**{n: getattr(torch, n) for n in ("int8", "uint8", "int32", "float32", "bfloat16", "float16", "float8_e4m3fn")},
                  "codes": {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}})   # tensors of the host stand for the device's
def no(f):
    try:
        f()
    except binding.EnsiError:
        return
    raise AssertionError("not refused")
x, gain = torch.zeros(4, 64), torch.ones(64)
ctx.clear_norm(x, gain)
no(lambda: ctx.clear_norm(x[0], gain))
no(lambda: ctx.clear_norm(x, gain.half()))
no(lambda: ctx.clear_norm(x, gain[:32]))
no(lambda: ctx.clear_norm(x.T, torch.ones(4)))
no(lambda: ctx.clear_norm(x, gain, residual=x[:2]))
no(lambda: ctx.clear_norm(x, gain, residual=x.double()))
no(lambda: ctx.clear_norm(x, gain, codes=torch.zeros(4, 128, dtype=torch.int8)[:, ::2]))
no(lambda: ctx.clear_norm(x.double(), gain.double()))
no(lambda: ctx.clear_norm(x, gain, codes=torch.zeros(4, 64, dtype=torch.uint8)))
w = ctx.clear_weights_prepare(np.zeros((64, 16), dtype=np.int8), np.ones(16))
codes, scales = torch.zeros(3, 64, dtype=torch.int8), torch.ones(3)
assert ctx.clear_matmul(w, codes, scales, dtype=torch.bfloat16).shape == (3, 16)
no(lambda: ctx.clear_matmul(w, codes[:, :32], scales, dtype=torch.bfloat16))
no(lambda: ctx.clear_matmul(w, codes, scales[:2], dtype=torch.bfloat16))
no(lambda: ctx.clear_matmul(w, codes, scales.half(), dtype=torch.bfloat16))
no(lambda: ctx.clear_matmul(w, codes, scales, torch.zeros(3, 17)))
no(lambda: ctx.clear_matmul(w, codes, scales, dtype=torch.int32))
k, s = torch.zeros(5, 2, 32, 64, dtype=torch.uint8), torch.zeros(5, 2, 2)
cache = ctx.clear_cache(k, k.clone(), s, s.clone())
no(lambda: ctx.clear_cache(k, k, s, s.clone()))
no(lambda: ctx.clear_cache(k.float(), k.float(), s, s))
no(lambda: ctx.clear_cache(k[0], k[0], s, s))
no(lambda: ctx.clear_cache(k, k[:4], s, s))
no(lambda: ctx.clear_cache(k, k.clone(), s[:, :, :1], s))
table, begin, lengths = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
kk, cos, q = torch.zeros(4, 2, 64), torch.zeros(9, 32), torch.zeros(4, 6, 64)
ctx.clear_append(cache, table, begin, lengths, kk, kk.clone(), cos, cos, q=q)
for bad in ((table.long(), begin, lengths), (table[0], begin, lengths), (table, begin[:2], lengths), (table, begin, lengths.float()), (table[:1], begin, lengths)):
    no(lambda: ctx.clear_append(cache, *bad, kk, kk, cos, cos))
    no(lambda: ctx.clear_attention(cache, *bad, q.half()))
no(lambda: ctx.clear_append(cache, table, begin, lengths, kk[:, :1], kk, cos, cos))
no(lambda: ctx.clear_append(cache, table, begin, lengths, kk, kk[:3], cos, cos))
no(lambda: ctx.clear_append(cache, table, begin, lengths, kk, kk.half(), cos, cos))
no(lambda: ctx.clear_append(cache, table, begin, lengths, kk, kk, cos, cos[:5]))
no(lambda: ctx.clear_append(cache, table, begin, lengths, kk, kk, cos[0], cos[0]))
no(lambda: ctx.clear_append(cache, table, begin, lengths, kk, kk, cos, cos, q=q[0]))
no(lambda: ctx.clear_append(cache, table, begin, lengths, kk, kk, cos, cos, q=q, q_out=q[:, :3]))
no(lambda: ctx.clear_append(cache, table, begin, lengths, torch.zeros(4, 2, 128)[:, :, ::2], kk, cos, cos))
ctx.clear_attention(cache, table, begin, lengths, q.half())
no(lambda: ctx.clear_attention(cache, table, begin, lengths, q))
no(lambda: ctx.clear_attention(cache, table, begin, lengths, q.half()[:, :5]))
no(lambda: ctx.clear_attention(cache, table, begin, lengths, q.half()[:, :, :32]))
no(lambda: ctx.clear_attention(cache, table, begin, lengths, q.half(), q.bfloat16()))
binding._TORCH = (lambda: 0, lambda at: 0, binding._TORCH[2])
no(lambda: ctx.clear_norm(x, gain))
""")
