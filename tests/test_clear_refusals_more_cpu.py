"""More of what the calls on clear activations refuse, without a GPU: numbers and arrays that no kernel should be launched on."""
from simhip import run
from test_clear_refusals_cpu import CACHE, PROGRAM, launches, names  # noqa: F401

NORM = PROGRAM + """
def norm(code=None, text="", **over):
    a = dict(x=at(65536), residual=0, gain=at(4096), sum_out=0, out=0, codes=at(4096), scales=at(4096), rows=4, x_stride=64, residual_stride=0, sum_stride=0, out_stride=0,
             d=64, type=1, eps=1e-5)
    a.update(over)
    rc = lib.ensi_clear_norm(ctx.h, binding._NORM.pack(*a.values(), 0), st)
    if code is None:
        assert rc == 0, lib.ensi_last_error(ctx.h)
    else:
        refused(rc, code, text)
"""


def test_norm_eps(tmp_path):
    calls = run(tmp_path, NORM + """
norm(eps=0.0)
norm(eps=3e38)
mark("bad")
norm(BADARG, "eps", eps=float("inf"))
""")
    assert len(launches(calls)) == 2


def test_norm_sum_into_an_input_whose_rows_lie_otherwise(tmp_path):
    """x and the residual begin at one address, their rows lie apart differently: a sum in place of either is read as the other's rows by other workgroups."""
    calls = run(tmp_path, NORM + """
x = at(65536)
norm(x=x, residual=x, residual_stride=64, sum_out=x, sum_stride=64)
norm(x=x, residual=x, residual_stride=128, x_stride=64, rows=1, sum_out=x, sum_stride=7)
mark("bad")
norm(BADARG, "overlaps", x=x, residual=x, residual_stride=128, sum_out=x, sum_stride=64)
norm(BADARG, "overlaps", x=x, residual=x, residual_stride=64, x_stride=128, sum_out=x, sum_stride=64)
norm(BADARG, "overlaps", x=x, residual=x, residual_stride=64, x_stride=128, sum_out=x, sum_stride=128)
norm(BADARG, "overlaps", x=x, residual=x + 128, residual_stride=64, sum_out=x, sum_stride=64)
norm(BADARG, "overlaps", x=x, residual=x + 128, residual_stride=64, sum_out=x + 128, sum_stride=64)
""")
    assert len(launches(calls)) == 2


SEQS = PROGRAM + CACHE + """
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
a = at(1 << 16)
"""


def test_append_rotates_in_place_beside_keys_and_values_only(tmp_path):
    """Queries of 256 elements, keys and values of 128, of two bytes: slices of one array whose columns meet would be rotated while they are read as keys."""
    calls = run(tmp_path, SEQS + """
wide = dict(q_stride=512, q_out_stride=512, k_stride=512, v_stride=512)
append(q=a, q_out=a, k=a + 512, v=a + 768, **wide)
append(q=a + 512, q_out=a + 512, k=a, v=a + 256, **wide)
append(q=a + 256, q_out=a + 256, k=a, v=a + 768, **wide)
append(q=a, q_out=at(1 << 16), k=a, v=a + 256, q_stride=512, k_stride=512, v_stride=512)     # (queries that are read only)
append(q=a, q_out=a + 512, k=a + 1024, v=a + 1280, q_stride=1024, q_out_stride=1024, k_stride=1024, v_stride=1024)  # rotated queries beside the others
append(q=a, q_out=a, k=a + 512, v=a + 768, tokens=1, q_stride=0, q_out_stride=0, k_stride=0, v_stride=0)
mark("bad")
append(BADARG, "k or v", q=a, q_out=a, k=a, v=a + 768, **wide)
append(BADARG, "k or v", q=a, q_out=a, k=a + 510, v=a + 768, **wide)
append(BADARG, "k or v", q=a, q_out=a, k=a + 512, v=a + 256, **wide)
append(BADARG, "k or v", q=a + 512, q_out=a + 512, k=a + 768 + 512, v=a, q_stride=384, q_out_stride=384, k_stride=384, v_stride=384)  # wraps round into the next token's queries
append(BADARG, "k or v", q=a, q_out=a, k=a + 512, v=a + 768, q_stride=512, q_out_stride=512, k_stride=256, v_stride=512)
append(BADARG, "k or v", q=a, q_out=a, k=a + 510, v=a + 768, tokens=1)
append(BADARG, "overlaps q", q=a, q_out=a + 510, k=a + 1024, v=a + 1280, q_stride=1024, q_out_stride=1024, k_stride=1024, v_stride=1024)
""")
    assert len(launches(calls)) == 6


def test_slices_of_one_array_are_apart(tmp_path):
    """Outputs beside their inputs in rows of one array."""
    calls = run(tmp_path, SEQS + NORM[len(PROGRAM):] + """
attention(q=a, out=a + 512, q_stride=512, out_stride=512)
attention(q=a + 512, out=a, q_stride=512, out_stride=512)
norm(x=a, x_stride=128, out=a + 128, out_stride=128)
norm(x=a, x_stride=256, residual=a + 128, residual_stride=256, sum_out=a + 256, sum_stride=256, out=a + 384, out_stride=256)
mark("bad")
attention(BADARG, "overlaps", q=a, out=a + 510, q_stride=512, out_stride=512)
attention(BADARG, "overlaps", q=a + 512, out=a + 2, q_stride=512, out_stride=512)
attention(BADARG, "overlaps", q=a, out=a + 512, q_stride=512, out_stride=768)
norm(BADARG, "overlaps", x=a, x_stride=128, out=a + 126, out_stride=128)
norm(BADARG, "overlaps", x=a, x_stride=256, residual=a + 128, residual_stride=256, sum_out=a + 256, sum_stride=256, out=a + 382, out_stride=256)
""")
    assert len(launches(calls)) == 4


def test_arrays_of_a_call_are_not_the_cache_s(tmp_path):
    """Nothing that a call writes, and nothing that an append reads, may lie in the cache that it writes or reads."""
    calls = run(tmp_path, SEQS + """
lib.ensi_clear_cache_free(kv)
parts = [at(1 << 20) for _ in range(4)]  # 10 pages of 2 heads, 32 tokens, 64 places: codes 40960 bytes, scales 160
rc, kv = wrap(k=parts[0], v=parts[1], ks=parts[2], vs=parts[3])
assert rc == 0
append(q=a, q_out=a)
attention(q=parts[0])   # (both only read)
mark("bad")
for p, size in zip(parts, (40960, 40960, 160, 160)):
    for at_ in (p, p + size - 2):
        append(BADARG, "cache", q=a, q_out=at_)
        append(BADARG, "cache", k=at_)
        append(BADARG, "cache", v=at_)
        append(BADARG, "cache", q=at_)
        attention(BADARG, "cache", out=at_)
    attention(out=p + size)
""")
    got = names(calls)
    assert sum("append" in n for n in got) == 1 and len([n for n in got if "attention" in n and "join" not in n]) == 5


BINDING = PROGRAM + """
import torch
binding._TORCH = (lambda: -1, lambda at: 0, {**{n: getattr(torch, n) for n in ("int8", "uint8", "int32", "float32", "bfloat16", "float16", "float8_e4m3fn")},
                  "codes": {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}})   # tensors of the host stand for the device's
def no(f, text=""):
    try:
        f()
    except binding.EnsiError as e:
        assert text in str(e), e
        return
    raise AssertionError("not refused")
x, gain = torch.zeros(4, 64), torch.ones(64)
w = ctx.clear_weights_prepare(np.zeros((64, 16), dtype=np.int8), np.ones(16))
codes, scales = torch.zeros(3, 64, dtype=torch.int8), torch.ones(3)
k, s = torch.zeros(5, 2, 32, 64, dtype=torch.uint8), torch.zeros(5, 2, 2)
cache = ctx.clear_cache(k, k.clone(), s, s.clone())
where = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
kk, cos, q = torch.zeros(4, 2, 64), torch.zeros(9, 32), torch.zeros(4, 6, 64)
"""


def test_tensors_that_require_a_gradient(tmp_path):
    """They are refused while gradients are recorded; without that they are tensors like others."""
    run(tmp_path, BINDING + """
leaf = lambda t: t.clone().requires_grad_()
bad = [lambda: ctx.clear_norm(leaf(x), gain), lambda: ctx.clear_norm(x, leaf(gain)), lambda: ctx.clear_norm(x, gain, residual=leaf(x)), lambda: ctx.clear_norm(leaf(x) * 2, gain),
       lambda: ctx.clear_matmul(w, codes, leaf(scales), dtype=torch.bfloat16),
       lambda: ctx.clear_append(cache, *where, leaf(kk), kk, cos, cos), lambda: ctx.clear_append(cache, *where, kk, leaf(kk), cos, cos), lambda: ctx.clear_append(cache, *where, kk, kk, cos, leaf(cos)),
       lambda: ctx.clear_append(cache, *where, kk, kk, cos, cos, q=leaf(q)), lambda: ctx.clear_attention(cache, *where, leaf(q.half())),
       lambda: ctx.clear_cache(k, k.clone(), leaf(s), s.clone())]
for f in bad:
    no(f, "requires a gradient")
with torch.no_grad():
    for f in bad:
        f()
with torch.inference_mode():
    for f in bad:
        f()
""")


def test_halves_of_pairs_of_arguments(tmp_path):
    """A place for rotated queries without queries, and one of cosines and sines, were passed over."""
    run(tmp_path, BINDING + """
no(lambda: ctx.clear_append(cache, *where, kk, kk, cos, cos, q_out=q), "q_out goes with q")
no(lambda: ctx.clear_append(cache, *where, kk, kk, None, cos), "cos with sin")
no(lambda: ctx.clear_append(cache, *where, kk, kk, cos, None), "cos with sin")
ctx.clear_append(cache, *where, kk, kk, None, None)
ctx.clear_append(cache, *where, kk, kk, cos, cos, q=q, q_out=q.clone())
""")


def test_numbers_names_and_handles_are_refused_as_such(tmp_path):
    """Numbers outside their type's range, unknown names, handles that are freed or another context's: the library's own error, with a message that is about it."""
    run(tmp_path, BINDING + """
h = q.half()
attend = lambda **over: ctx.clear_attention(cache, *where, h, **over)
no(lambda: attend(score="maximum"), "score")
no(lambda: ctx.clear_append(cache, *where, kk, kk, cos, cos, pairs="both"), "pairs")
for over in (dict(window=1 << 31), dict(window=2.5), dict(max_length=1 << 40), dict(max_new=-(1 << 40)), dict(cap=1e39), dict(bias=-1e39)):
    no(lambda: attend(**over), "range")
no(lambda: ctx.clear_append(cache, *where, kk, kk, cos, cos, max_new=1 << 33), "range")
no(lambda: ctx.clear_norm(x, gain, eps=1e39), "range")
no(lambda: ctx.clear_attention(cache, where[0], where[1], where[2][0], h), "lengths")
no(lambda: ctx.clear_append(cache, *where, kk[0, 0, 0], kk, cos, cos), "tokens")
no(lambda: ctx.clear_append(cache, *where, kk[0], kk, cos, cos), "tokens")
other = binding.Context(12, 36, 3, 37, 1, 1, 30)
no(lambda: other.clear_attention(cache, *where, h), "another context")
no(lambda: other.clear_append(cache, *where, kk, kk, cos, cos), "another context")
no(lambda: other.clear_matmul(w, codes, scales, dtype=torch.float32), "another context")
no(lambda: ctx.clear_norm(x, gain, eps=-1.0), "eps")  # (an error of another call before)
cache.free()
w.free()
no(lambda: ctx.clear_attention(cache, *where, h), "no cache")
no(lambda: ctx.clear_append(cache, *where, kk, kk, cos, cos), "no cache")
no(lambda: ctx.clear_matmul(w, codes, scales, dtype=torch.float32), "no weights")
no(lambda: cache.check(), "no cache")
""")
