"""What the calls of drafted decoding refuse, without a GPU: every wrong argument is answered with its code and a message before anything is launched, and good ones launch on the
stream that they are given."""
from simhip import run
from test_clear_refusals_cpu import launches, names
from test_clear_refusals_more_cpu import SEQS


def test_null_arguments(tmp_path):
    run(tmp_path, SEQS + """
n = None
assert lib.ensi_clear_sample(n, b"", n) == -1 and lib.ensi_clear_sample(ctx.h, n, n) == -1
assert lib.ensi_clear_accept(n, b"", n) == -1 and lib.ensi_clear_accept(ctx.h, n, n) == -1
assert lib.ensi_clear_append_tree(n, n, b"", n, n) == -1 and lib.ensi_clear_append_tree(ctx.h, kv, b"", n, n) == -1 and lib.ensi_clear_append_tree(ctx.h, kv, n, 4096, n) == -1
assert lib.ensi_clear_attention_tree(n, n, b"", n, n) == -1 and lib.ensi_clear_attention_tree(ctx.h, kv, b"", n, n) == -1 and lib.ensi_clear_attention_tree(ctx.h, n, b"", 4096, n) == -1
assert lib.ensi_clear_keep(n, n, 0, b"", n) == -1 and lib.ensi_clear_keep(ctx.h, n, 1, b"", n) == -1 and lib.ensi_clear_keep(ctx.h, b"", 1, n, n) == -1
assert lib.ensi_clear_fork(n, n, 0, b"", n) == -1 and lib.ensi_clear_fork(ctx.h, n, 1, b"", n) == -1 and lib.ensi_clear_fork(ctx.h, b"", 1, n, n) == -1
""")


def test_sample(tmp_path):
    calls = run(tmp_path, SEQS + """
def sample(code=None, text="", **over):
    a = dict(logits=at(1 << 16), uniform=at(64), temperature=at(64), top_k=at(64), top_p=at(64), min_p=at(64), out=at(64), rows=4, stride=1000, vocab=1000, type=1, t=1.0, k=0, p=1.0, m=0.0)
    a.update(over)
    check(lib.ensi_clear_sample(ctx.h, binding._SAMPLE.pack(*a.values()), st), code, text)
x, o = at(1 << 16), at(4096)
mark("good")
sample()
sample(rows=0, logits=0, uniform=0, out=0)
sample(temperature=0, top_k=0, top_p=0, min_p=0, t=0.0, k=-5, p=7.0, m=-2.0)
sample(rows=1, stride=0)
sample(temperature=at(64), t=-1.0)  # not looked at beside an array
sample(logits=x, out=x + 2000, rows=1)
mark("bad")
sample(BADARG, "type", type=3)
sample(SHAPE, "rows", rows=-1)
sample(SHAPE, "rows", rows=(1 << 20) + 1)
sample(SHAPE, "logits", vocab=0, stride=0)
sample(SHAPE, "logits", vocab=(1 << 24) + 1, stride=1 << 25)
sample(SHAPE, "overlap", stride=999)
sample(SHAPE, "overlap", stride=-1000)
for name in ("logits", "uniform", "out"):
    sample(BADARG, "needed", **{name: 0})
for t in (-1.0, float("inf"), float("nan")):
    sample(BADARG, "temperature", temperature=0, t=t)
sample(BADARG, "top_p", top_p=0, p=float("nan"))
sample(BADARG, "min_p", min_p=0, m=float("nan"))
sample(BADARG, "overlaps", logits=x, out=x + 1998, rows=1)
sample(BADARG, "overlaps", logits=x, out=x + 2 * 3999)
for name in ("uniform", "temperature", "top_k", "top_p", "min_p"):
    sample(BADARG, "overlaps", out=o, **{name: o + 12})
""")
    assert len(launches(calls)) == 5 and all(c[1] == "0x1000" for c in launches(calls))


def test_rows_are_split_where_they_are_few_and_long(tmp_path):
    """Four launches on one stream where a row is split (three without top_k and top_p), one otherwise."""
    calls = run(tmp_path, SEQS + """
def sample(rows, vocab, p=1.0):
    u, out = at(1 << 14), at(1 << 14)
    a = (at(rows * vocab * 2), u, 0, 0, 0, 0, out, rows, vocab, vocab, 1, 1.0, 0, p, 0.0)
    check(lib.ensi_clear_sample(ctx.h, binding._SAMPLE.pack(*a), st), None, "")
sample(1, 32000)
sample(1, 128000, 0.9)
sample(2, 128000)
sample(2000, 128000, 0.9)
""")
    kinds = [n.split("k_clear_sample")[1].split("ILi")[0] for n in names(calls)]
    assert kinds == ["", "_most", "_bins", "_gather", "_finish", "_most", "_bins", "_finish", ""]
    assert all(c[1] == "0x1000" for c in launches(calls))


def test_trees(tmp_path):
    calls = run(tmp_path, SEQS + """
parents, o = at(64), at(1 << 16)
def tree(which, code=None, text="", parents=parents, **over):
    s = seqs(over)
    if which == "append":
        a = dict(q=at(1 << 16), k=at(1 << 16), v=at(1 << 16), q_out=at(1 << 16), cos=at(1 << 16), sin=at(1 << 16), q_stride=256, q_out_stride=256, k_stride=128, v_stride=128, q_heads=4, rot=64,
                 positions=100, pairs=0, type=1)
        a.update(over)
        rc = lib.ensi_clear_append_tree(ctx.h, kv, binding._APPEND.pack(*s, *a.values(), 0), parents, st)
    else:
        a = dict(q=at(1 << 16), out=at(1 << 16), q_stride=256, out_stride=256, q_heads=4, type=1, score=0, window=0, max_length=100, cap=0.0, bias=0.0)
        a.update(over)
        rc = lib.ensi_clear_attention_tree(ctx.h, kv, binding._ATTENTION.pack(*s, *a.values(), 0), parents, st)
    check(rc, code, text)
mark("good")
for which in ("append", "attention"):
    tree(which)
    tree(which, max_new=64, tokens=100)
    tree(which, tokens=0)
mark("bad")
for which in ("append", "attention"):
    tree(which, BADARG, "parents", parents=None)
    tree(which, SHAPE, "trees of up to 64", max_new=65)
    tree(which, SHAPE, "sequences", seqs=-1)
    tree(which, BADARG, "table", table=0)
    tree(which, SHAPE, "heads", q_heads=0)
tree("attention", BADARG, "parents", out=o, parents=o + 8)
tree("append", BADARG, "parents", q_out=o, parents=o + 8)
tree("attention", SHAPE, "query heads", q_heads=3)
tree("attention", BADARG, "type", type=0)
""")
    made = names(calls)
    assert len([n for n in made if "k_clear_append" in n]) == 2 and all(n.endswith("Lb1EEv10AppendView") for n in made if "k_clear_append" in n)
    assert all("attention_tree" in n for n in made if "append" not in n) and all(c[1] == "0x1000" for c in launches(calls))


def test_accept(tmp_path):
    calls = run(tmp_path, SEQS + """
def accept(code=None, text="", **over):
    a = dict(begin=at(64), parents=at(64), drafted=at(64), sampled=at(64), path=at(4096), count=at(64), following=at(64), tokens=10, path_stride=5, seqs=3, max_new=5)
    a.update(over)
    check(lib.ensi_clear_accept(ctx.h, binding._ACCEPT.pack(*a.values()), st), code, text)
x = at(4096)
mark("good")
accept()
accept(parents=0)
accept(seqs=0, begin=0, path=0)
accept(max_new=0, path=0, tokens=0, drafted=0, sampled=0)
accept(seqs=1, path_stride=0)
mark("bad")
accept(SHAPE, "sequences", seqs=-1)
accept(SHAPE, "sequences", seqs=65536)
accept(SHAPE, "at most", max_new=65, path_stride=65)
accept(SHAPE, "at most", max_new=-1)
accept(SHAPE, "new tokens", tokens=-1)
for name in ("begin", "drafted", "sampled", "path", "count", "following"):
    accept(BADARG, "null", **{name: 0})
accept(SHAPE, "overlap", path_stride=4)
for name in ("begin", "parents", "drafted", "sampled"):
    accept(BADARG, "input", path=x, **{name: x + 16})
    accept(BADARG, "input", count=x, **{name: x + 8})
accept(BADARG, "outputs", path=x, count=x + 40)
accept(BADARG, "outputs", following=x, count=x + 8)
""")
    assert len(launches(calls)) == 4


KEEP = SEQS + """
import struct
rc, other = wrap()
assert rc == 0
hands = lambda *h: struct.pack("%dQ" % len(h), *[x if isinstance(x, int) else x.value for x in h])
"""


def test_keep(tmp_path):
    calls = run(tmp_path, KEEP + """
def keep(code=None, text="", caches=None, **over):
    s = seqs(over)
    a = dict(path=at(4096), count=at(64), path_stride=4)
    a.update(over)
    h = hands(*(caches or [kv]))
    check(lib.ensi_clear_keep(ctx.h, h, len(h) // 8, binding._KEEP.pack(*s, *a.values()), st), code, text)
mark("good")
keep()
keep(caches=[kv, other])
keep(tokens=0, path=0)
keep(seqs=1, path_stride=0)
mark("bad")
check(lib.ensi_clear_keep(ctx.h, hands(kv), 0, binding._KEEP.pack(*seqs({}), 1, 1, 4), st), SHAPE, "caches")
check(lib.ensi_clear_keep(ctx.h, hands(kv), 1025, binding._KEEP.pack(*seqs({}), 1, 1, 4), st), SHAPE, "caches")
keep(BADARG, "no cache", caches=[kv, 0])
keep(BADARG, "twice", caches=[kv, other, kv])
keep(SHAPE, "trees of up to 64", max_new=65, path_stride=65)
keep(SHAPE, "sequences", seqs=70000)
keep(BADARG, "table", lengths=0)
keep(BADARG, "path and count", path=0)
keep(BADARG, "path and count", count=0)
keep(SHAPE, "overlap", path_stride=3)
second = binding.Context(12, 36, 3, 37, 1, 1, 30)
rc = lib.ensi_clear_keep(second.h, hands(kv), 1, binding._KEEP.pack(*seqs({}), at(64), at(64), 4), st)
assert rc == BADARG and b"another context" in lib.ensi_last_error(second.h)
""")
    assert len(launches(calls)) == 3


def test_fork(tmp_path):
    calls = run(tmp_path, KEEP + """
def fork(code=None, text="", caches=None, **over):
    a = dict(table=at(4096), lengths=at(64), source=at(64), fresh=at(64), table_out=at(4096), lengths_out=at(64), table_stride=8, out_stride=8, seqs=3, rows=5, table_width=8)
    a.update(over)
    h = hands(*(caches or [kv]))
    check(lib.ensi_clear_fork(ctx.h, h, len(h) // 8, binding._FORK.pack(*a.values(), 0), st), code, text)
x = at(4096)
mark("good")
fork()
fork(caches=[kv, other])
fork(rows=0, source=0)
fork(seqs=0, table=0, lengths=0)
mark("bad")
fork(BADARG, "twice", caches=[other, other])
fork(SHAPE, "rows", rows=-1)
fork(SHAPE, "rows", rows=65536)
fork(SHAPE, "sequences", seqs=65536)
fork(SHAPE, "pages", table_width=0)
for name in ("table", "lengths", "source", "fresh", "table_out", "lengths_out"):
    fork(BADARG, "null", **{name: 0})
fork(SHAPE, "overlap", table_stride=7)
fork(SHAPE, "overlap", out_stride=7)
fork(BADARG, "input", table=x, table_out=x)
fork(BADARG, "input", table=x, lengths_out=x + 92)
for name in ("lengths", "source", "fresh"):
    fork(BADARG, "input", table_out=x, **{name: x + 4})
fork(BADARG, "outputs", table_out=x, lengths_out=x + 156)
""")
    assert len(launches(calls)) == 3


def test_binding(tmp_path):
    """Tensors of the wrong kind are refused by name before a call is made."""
    import pytest
    torch = pytest.importorskip("torch")
    from paper_2509_09424_amd import binding

    class Ctx(binding.Context):
        def __init__(self):
            self.lib = self.h = None

    ctx, E = Ctx(), binding.EnsiError
    names = {n: getattr(torch, n) for n in ("int8", "uint8", "int32", "float32", "bfloat16", "float16", "float8_e4m3fn")}
    names["codes"] = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    before, binding._TORCH = binding._TORCH, (lambda: -1, lambda at: 0, names)
    try:
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
        x, u = torch.zeros(3, 10), torch.zeros(3)
        for match, call in (
            ("logits", lambda: ctx.clear_sample(x[0], u)), ("logits", lambda: ctx.clear_sample(x.double(), u)), ("uniform", lambda: ctx.clear_sample(x, u[:2])), ("uniform", lambda: ctx.clear_sample(x, u.double())),
            ("temperature", lambda: ctx.clear_sample(x, u, temperature=i32(3))), ("top_k", lambda: ctx.clear_sample(x, u, top_k=u)), ("top_p", lambda: ctx.clear_sample(x, u, top_p=torch.zeros(1))),
            ("not a number", lambda: ctx.clear_sample(x, u, temperature="warm")), ("not a number", lambda: ctx.clear_sample(x, u, top_k=1 << 40)), ("not a number", lambda: ctx.clear_sample(x, u, top_k=1.5)),
            ("out", lambda: ctx.clear_sample(x, u, out=torch.zeros(3, dtype=torch.int64))), ("logits", lambda: ctx.clear_sample(x[:, ::2], u)), ("gradient", lambda: ctx.clear_sample(x.clone().requires_grad_(), u)),
            ("begin", lambda: ctx.clear_accept(i32(0), None, i32(4), i32(4))), ("sampled", lambda: ctx.clear_accept(i32(2), None, i32(4), i32(3))), ("parents", lambda: ctx.clear_accept(i32(2), i32(4).long(), i32(4), i32(4))),
            ("path", lambda: ctx.clear_accept(i32(2), None, i32(4), i32(4), path=i32(2, 4))), ("caches", lambda: ctx.clear_keep([], i32(1, 1), i32(2), i32(1), i32(1), i32(1))),
            ("caches", lambda: ctx.clear_keep(None, i32(1, 1), i32(2), i32(1), i32(1, 4), i32(1))), ("caches", lambda: ctx.clear_fork([None], i32(1, 1), i32(1), i32(1), i32(1))),
        ):
            with pytest.raises(E, match=match):
                call()
    finally:
        binding._TORCH = before


def test_a_few_of_every_rows_tokens_take_a_launch_less(tmp_path):
    calls = run(tmp_path, SEQS + """
u, out, x = at(64), at(64), at(2 * 128000 * 2)
for t, k, each in ((0.8, 50, 0), (0.8, 3584, 0), (0.8, 3585, 0), (0.0, 50, 0), (0.8, 50, at(64))):
    check(lib.ensi_clear_sample(ctx.h, binding._SAMPLE.pack(x, u, 0, each, 0, 0, out, 2, 128000, 128000, 1, t, k, 0.9, 0.0), st), None, "")
""")
    kinds = "".join({"_most": "m", "_bins": "b", "_gather": "g", "_finish": "f"}[n.split("k_clear_sample")[1].split("ILi")[0]] for n in names(calls))
    assert kinds == "mgf" * 2 + "mbgf" * 3  # (7 workgroups to a row, 512 tokens each)
