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
