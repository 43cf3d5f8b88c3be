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
