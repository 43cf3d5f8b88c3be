"""Sampling against its definition in 64 bits: tokens are whole numbers and have to be equal.  A running sum in 64 bits is off by 2^-53 of its terms, and the library's by 2^-46 of the
largest weight for each, so the two differ where a border lies that near to a sum, which it does for none of these inputs."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    from paper_2509_09424_amd import Context
    c = Context(12, 36, 3, 37, 1, 1, 30)
    yield c
    c.close()


def reference(x, u, t, k, p, m):
    """One row, from the definition."""
    x = x.astype(np.float64)
    if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any() or not 0 <= t < np.inf or any(map(math.isnan, (u, p, m))):
        return -1
    if t == 0:
        return int(np.argmax(x))
    with np.errstate(over="ignore", under="ignore"):
        e = (x - x.max()) / t
        w = np.exp(e)
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if k > 0:
        order = order[:k]
    if p < 1:
        run = np.cumsum(w[order])
        order = order[:1 + int(np.sum(run[:-1] < p * run[-1]))] if p > 0 else order[:1]
    # w >= m by their logarithms: exp(-1e-38) is below 1, but 1 in 64 bits
    left = np.sort(order[e[order] >= math.log(min(m, 1.0))]) if m > 0 else np.sort(order)
    run = np.cumsum(w[left])
    return int(left[min(int(np.sum(run <= min(max(u, 0.0), 1.0) * run[-1])), len(left) - 1)])


def check(ctx, x, u, t, k, p, m, pad=0):
    """x: [rows][vocab] of a type; the others lists or arrays of numbers, rounded to 32 bits."""
    rows, vocab = x.shape
    wide = torch.full((rows, vocab + pad), 99.0, dtype=x.dtype)
    wide[:, :vocab] = x
    u, t, p, m = (np.broadcast_to(np.asarray(a, dtype=np.float32), rows) for a in (u, t, p, m))
    k = np.broadcast_to(np.asarray(k, dtype=np.int32), rows)
    dev = lambda a: torch.from_numpy(a.copy()).cuda()  # noqa: E731
    logits = wide.cuda()[:, :vocab]
    got = ctx.clear_sample(logits, dev(u), temperature=dev(t), top_k=dev(k), top_p=dev(p), min_p=dev(m))
    numbers = x.float().numpy()
    want = [reference(numbers[r], float(u[r]), float(t[r]), int(k[r]), float(p[r]), float(m[r])) for r in range(rows)]
    got = got.cpu().tolist()
    assert got == want, [(r, g, w) for r, (g, w) in enumerate(zip(got, want)) if g != w][:10]
    return logits


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows, vocab, pad", [(1, 1, 0), (5, 2, 1), (9, 7, 0), (40, 63, 0), (40, 65, 3), (40, 255, 1), (40, 511, 0), (40, 513, 0), (40, 4099, 1), (30, 8192, 0), (30, 32000, 8), (12, 65537, 0), (6, 131072, 0),
                                              (6, 131073, 5), (3, 200003, 0)])
def test_settings_of_every_kind(ctx, kind, rows, vocab, pad):
    rng = np.random.default_rng(rows * vocab)
    x = torch.from_numpy(rng.standard_normal((rows, vocab)) * rng.uniform(0.01, 4, (rows, 1))).to(TYPES[kind])
    check(ctx, x, rng.random(rows), rng.choice([0, 0.3, 0.7, 1, 1, 2.5], rows), rng.choice([0, 0, 1, 2, 17, 300, 2000, 5000, vocab - 1, vocab, vocab + 5], rows), rng.choice([1, 1, 0.05, 0.5, 0.9, 0.99, 0.0], rows),
          rng.choice([0, 0, 1e-6, 0.01, 0.3, 1.0], rows), pad)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_equal_logits(ctx, kind):
    """Among equal logits the lower index comes first: cuts within them by top_k and top_p, and rows of nothing else."""
    rng = np.random.default_rng(3)
    rows, vocab = 48, 10007
    x = np.round(rng.standard_normal((rows, vocab)) * 2) / 2
    x[::4] = 1.25
    x[1::4, :] = np.where(rng.random((rows // 4, vocab)) < 0.5, 0.0, -0.0)  # zeros of either sign are equal
    x[2::4] = np.where(rng.random((rows // 4, vocab)) < 0.01, 3.0, x[2::4])
    check(ctx, torch.from_numpy(x).to(TYPES[kind]), rng.random(rows), rng.choice([0, 1, 1, 0.1], rows), rng.choice([0, 1, 100, 3500, 9999], rows), rng.choice([1, 0.3, 0.77], rows), rng.choice([0, 0.9, 1], rows))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_masked_logits(ctx, kind):
    """-inf among the logits is never taken; a row of nothing else, NaN and +inf have no distribution."""
    rng = np.random.default_rng(4)
    x = rng.standard_normal((24, 3000)).astype(np.float32)
    x[rng.random(x.shape) < 0.7] = -np.inf
    x[0] = -np.inf
    x[1, 5] = np.nan
    x[2, 2999] = np.inf
    x[3] = -np.inf
    x[3, 2998] = -5.0
    x[4, ::2] = -np.inf
    x[5, 0], x[5, 1] = np.nan, -np.nan
    x[6] = -np.inf
    x[6, 7:9] = -3e38 if kind == "f32" else -3e37
    for t in (1.0, 0.0):
        check(ctx, torch.from_numpy(x).to(TYPES[kind]), rng.random(24), t, [0, 0, 0, 0, 5, 0] * 4, 1.0, 0.0)
        check(ctx, torch.from_numpy(x).to(TYPES[kind]), rng.random(24), t, 0, 0.8, 0.01)


def test_numbers_at_the_ends_of_their_ranges(ctx):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((40, 2500)).astype(np.float32) * 3
    x[10:20] *= 1e37
    x[20:30] *= 1e-30
    x[35] = -x[35] ** 2 - 1e6
    last = 1 - 2.0 ** -24
    t = [1, 1e-38, 1e-45, 3e38, 1e5] * 8
    u = [last, 2.0 ** -24, 0.25, 0.5, last, 0.999, 0.1] * 5 + [last] * 5
    check(ctx, torch.from_numpy(x), u, t, [0, 3, 0, 0, 2500, 1] * 6 + [0] * 4, [1, 0.5, 1, 2.5, 1e-30, -1, last] * 5 + [1] * 5, [0, 0, 1e-40, 1, 7, -3] * 6 + [0] * 4)
    # what has no distribution
    nan, inf = math.nan, math.inf
    check(ctx, torch.from_numpy(x[:9]), [0.5, 0.5, 0.5, nan, 0.5, 0.5, 0.5, 0.5, 0.5], [-1, nan, inf, 1, 1, 1, 1, 0, -0.0], 0, [1, 1, 1, 1, nan, 1, 0.5, 1, 1], [0, 0, 0, 0, 0, nan, 0, 0, 0])
    # random numbers outside of [0, 1) count as the nearest inside
    check(ctx, torch.from_numpy(x[:6]), [1.0, 1.5, inf, 1.0, 2.0, 1.0], 1, [0, 5, 0, 2, 0, 1], [1, 1, 0.9, 1, 1, 1], 0)
    low = ctx.clear_sample(torch.from_numpy(x[:2]).cuda(), torch.tensor([-1.0, 0.0], device="cuda"), top_k=4).cpu().tolist()
    assert low == [int(np.sort(np.argsort(-x[r])[:4])[0]) for r in range(2)]


def test_numbers_for_all_rows_and_frequencies(ctx):
    """Parameters as numbers; evenly spaced random numbers give every token its share."""
    p = np.array([0.5, 0.25, 0.125, 0.0625, 0.0625])
    x = torch.from_numpy(np.log(p)).float().repeat(4096, 1).cuda()
    u = (torch.arange(4096, device="cuda") + 0.5) / 4096
    got = ctx.clear_sample(x, u).cpu()
    assert got.bincount().tolist() == [2048, 1024, 512, 256, 256]
    got = ctx.clear_sample(x, u, top_k=2, temperature=0.5).cpu()  # 0.8 and 0.2
    assert abs(int((got == 0).sum()) - 4096 * 0.8) <= 1 and set(got.tolist()) == {0, 1}
    got = ctx.clear_sample(x, u, top_p=0.8, min_p=0.3).cpu()
    assert set(got.tolist()) == {0, 1}
    assert ctx.clear_sample(x, u, temperature=0).cpu().eq(0).all()
    out = torch.full((4096,), 7, dtype=torch.int32, device="cuda")
    assert ctx.clear_sample(x, u, out=out) is out and torch.equal(out.cpu(), ctx.clear_sample(x, u).cpu())


def test_rows_past_32_bits_and_the_largest_vocabulary(ctx):
    """Rows that begin beyond 2^31 elements, and 2^22 + 3 logits in a row."""
    x = torch.full((3, 1 << 30), -math.inf, dtype=torch.bfloat16, device="cuda")[:, :5000]
    x[:] = torch.randn(3, 5000, generator=torch.Generator().manual_seed(1)).cuda()
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    want = [reference(x[r].float().cpu().numpy(), float(u[r]), 1.0, 0, 1.0, 0.0) for r in range(3)]
    assert ctx.clear_sample(x, u).cpu().tolist() == want
    del x
    rng = np.random.default_rng(8)
    check(ctx, torch.from_numpy(rng.standard_normal((3, (1 << 22) + 3)).astype(np.float32)), [0.3, 0.6, 0.99], [1, 0.7, 0.2], [0, 100000, 0], [1, 0.9, 0.4], 0)


def test_a_captured_call_follows_its_inputs(ctx):
    rng = np.random.default_rng(9)
    x, u = torch.empty(7, 5000, device="cuda"), torch.empty(7, device="cuda")
    fill = lambda: (x.copy_(torch.from_numpy(rng.standard_normal((7, 5000)).astype(np.float32))), u.copy_(torch.from_numpy(rng.random(7).astype(np.float32))))  # noqa: E731
    fill()
    out = torch.zeros(7, dtype=torch.int32, device="cuda")
    run = lambda: ctx.clear_sample(x, u, temperature=0.8, top_k=50, top_p=0.9, out=out)  # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        fill()
        graph.replay()
        got = out.cpu().tolist()
        assert got == ctx.clear_sample(x, u, temperature=0.8, top_k=50, top_p=0.9).cpu().tolist()
        numbers, un = x.cpu().numpy(), u.cpu().numpy()
        assert got == [reference(numbers[r], float(un[r]), float(np.float32(0.8)), 50, float(np.float32(0.9)), 0.0) for r in range(7)]


@pytest.mark.parametrize("kind, vocab", [("bf16", 70001), ("f32", 40000), ("f16", 128000), ("bf16", 500)])
def test_numbers_for_all_rows_are_arrays_of_them(ctx, kind, vocab):
    """Which passes a call makes depends on what it knows of the rows; the tokens do not."""
    rng = np.random.default_rng(vocab)
    x = torch.from_numpy(rng.standard_normal((5, vocab)).astype(np.float32) * 3).to(TYPES[kind])
    x[3] = -math.inf
    x[4, :vocab // 2] = 2.0  # equal ones, more than there is room for
    u = rng.random(5).astype(np.float32)
    for t, k, p, m in ((0.8, 50, 0.95, 0.0), (1.0, 1, 1.0, 0.0), (1.3, 2000, 0.9, 0.01), (1.3, 5000, 1.0, 0.0), (0.0, 50, 0.9, 0.0), (0.7, vocab, 0.9, 0.0), (0.7, vocab - 1, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (0.7, -3, 1.0, 0.1)):
        logits = check(ctx, x, u, t, k, p, m)
        numbers = [reference(x[r].float().numpy(), float(u[r]), *(float(np.float32(a)) if i != 1 else a for i, a in enumerate((t, k, p, m)))) for r in range(5)]
        assert ctx.clear_sample(logits, torch.from_numpy(u).cuda(), temperature=t, top_k=k, top_p=p, min_p=m).cpu().tolist() == numbers, (t, k, p, m)
