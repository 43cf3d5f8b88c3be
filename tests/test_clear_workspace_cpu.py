"""The workspace of the calls on clear activations where there is no memory for it, without a GPU: sampling goes on without it, and does not ask again in every call; a cache, which needs it, does."""
import subprocess

import simhip
from test_clear_refusals_cpu import launches
from test_clear_refusals_more_cpu import PROGRAM

FULL = simhip.SOURCE.replace("""hipError_t hipMalloc(void **p, size_t n) {""", """static bool full = false;
void simhip_full(int on) { full = on; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n) {
    if (full && n >= 64 << 20) { LOG("refused"); *p = nullptr; return hipErrorOutOfMemory; }""")


def run(tmp_path, body):
    (tmp_path / "simhip.cpp").write_text(FULL)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", str(tmp_path / "simhip.cpp"), "-o", str(tmp_path / "libsimhip.so")], check=True)
    return simhip.run(tmp_path, PROGRAM + """
def sample(rows=2, vocab=128000):
    x, u, out = at(64), at(rows * vocab * 2), at(1 << 14)
    rc = lib.ensi_clear_sample(ctx.h, binding._SAMPLE.pack(x, u, 0, 0, 0, 0, out, rows, vocab, vocab, 1, 1.0, 0, 0.9, 0.0), st)
    assert rc == 0, lib.ensi_last_error(ctx.h)
def cache():
    kv = ctypes.c_void_p()
    rc = lib.ensi_clear_cache_wrap(ctx.h, *(ctypes.c_void_p(at(1 << 16)) for _ in range(4)), 2, 2, 16, 64, ctypes.byref(kv))
    return rc
""" + body)


def test_refused_memory_is_asked_for_once(tmp_path):
    calls = run(tmp_path, """
sim.simhip_full(1)
for _ in range(5):
    sample()
""")
    asked = [i for i, c in enumerate(calls) if c[0] == "refused"]
    first = next(i for i, c in enumerate(calls) if c[0] == "launch" and "k_clear_sample" in c[2])
    assert asked and all(i < first for i in asked)
    assert len(launches(calls)) == 5  # one kernel each


def test_a_cache_asks_again(tmp_path):
    calls = run(tmp_path, """
sim.simhip_full(1)
sample()
assert cache() == -5, lib.ensi_last_error(ctx.h)  # no memory
sample()
sim.simhip_full(0)
sample()
assert cache() == 0
mark("made")
sample()
""")
    made = [c[0] for c in calls].index("mark")
    assert len(launches(calls[:made])) == 3 and len(launches(calls[made:])) == 4


def test_the_first_call_makes_it(tmp_path):
    calls = run(tmp_path, """
mark("first")
sample()
mark("second")
sample()
""")
    first, second = (i for i, c in enumerate(calls) if c[0] == "mark")
    assert [c[0] for c in calls[first:second]].count("alloc") == 1 and [c[0] for c in calls[second:]].count("alloc") == 0 and len(launches(calls)) == 8
