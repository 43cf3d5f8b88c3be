"""The calls on the caches of many layers refuse caches that have memory in common, without a GPU: what one wave of such a call writes, another would read, with no order between them."""
import pytest

from simhip import run
from test_clear_drafted_refusals_cpu import KEEP
from test_clear_refusals_cpu import launches

# arrays of a cache of 3 pages, 2 heads, 32 tokens, 64 places: 12288 codes, 12 scales
APART = KEEP + """
K, S = 3 * 2 * 32 * 64, 3 * 2 * 2 * 4
def cache(**over):
    a = dict(k=at(1 << 16), v=at(1 << 16), ks=at(1 << 16), vs=at(1 << 16))
    a.update(over)
    h = ctypes.c_void_p()
    rc = lib.ensi_clear_cache_wrap(ctx.h, *(ctypes.c_void_p(a[n]) for n in ("k", "v", "ks", "vs")), 3, 2, 32, 64, ctypes.byref(h))
    assert rc == 0, lib.ensi_last_error(ctx.h)
    return h
def both(code, text, *caches):
    h = hands(*caches)
    check(lib.ensi_clear_keep(ctx.h, h, len(caches), binding._KEEP.pack(*seqs({}), at(4096), at(64), 4), st), code, text)
    check(lib.ensi_clear_fork(ctx.h, h, len(caches), binding._FORK.pack(at(4096), at(64), at(64), at(64), at(4096), at(64), 8, 8, 3, 5, 8, 0), st), code, text)
x, s = at(1 << 20), at(1 << 20)
where[0] += 1 << 20
"""


def test_caches_side_by_side(tmp_path):
    """Neighbours in one allocation, in any order, and as many as a call takes."""
    calls = run(tmp_path, APART + """
parts = [cache(k=x + 2 * i * K, v=x + (2 * i + 1) * K, ks=s + 2 * i * S, vs=s + (2 * i + 1) * S) for i in range(5)]
both(None, "", *parts)
both(None, "", *[parts[i] for i in (3, 0, 4, 2, 1)])
both(None, "", *[cache() for _ in range(1024)])
""")
    assert len(launches(calls)) == 2 * (1 + 1 + 32)


@pytest.mark.parametrize("first, second", [
    ("k=x", "k=x"), ("k=x", "k=x + K - 64"), ("k=x + K - 16", "k=x"), ("v=x", "v=x"), ("k=x", "v=x + 2048"), ("v=x + 2048", "k=x"), ("ks=s", "ks=s"), ("vs=s", "vs=s + S - 4"), ("ks=s + 4", "vs=s"), ("k=x", "vs=x + 64")])
def test_caches_that_meet(tmp_path, first, second):
    calls = run(tmp_path, APART + """
one, two = cache(%s), cache(%s)
both(BADARG, "overlap", one, two)
both(BADARG, "overlap", two, cache(), one)
""" % (first, second))
    assert not launches(calls)
