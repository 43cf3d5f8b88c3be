"""Sampling with a top_k of thousands in rows that are split over workgroups: the tokens, and that such rows go the way of candidates and not that of a search in the row itself."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_clear_sample import TYPES, check, ctx  # noqa: E402, F401

pytestmark = pytest.mark.gpu

TOP_K = [3000, 3300, 3584, 3585, 3800, 4000, 4095, 4096]


@pytest.mark.parametrize("kind, vocab", [("bf16", 131072), ("f32", 200003), ("f16", 128000), ("bf16", 98304), ("f32", 50000)])
def test_thousands_of_candidates(ctx, kind, vocab):  # noqa: F811
    rng = np.random.default_rng(vocab)
    x = torch.from_numpy(rng.standard_normal((8, vocab)).astype(np.float32) * 2).to(TYPES[kind])
    check(ctx, x, rng.random(8), [1, 0.7, 1.5, 1, 2, 1, 0.5, 1], TOP_K, [0.95, 1, 0.9, 0.999, 1, 1, 0.5, 0.97], [0, 0, 0, 0.001, 0.01, 0, 0, 0])
    for k in TOP_K:
        got = ctx.clear_sample(x.cuda(), torch.full((8,), 0.7, device="cuda"), top_k=k, top_p=0.99).tolist()
        assert got == ctx.clear_sample(x.cuda(), torch.full((8,), 0.7, device="cuda"), top_k=torch.full((8,), k, dtype=torch.int32, device="cuda"), top_p=0.99).tolist()


@pytest.mark.parametrize("large, of", [(3000, 16384), (4090, 16384), (4500, 16384), (7000, 16384), (9000, 16384), (6000, 32768)])
def test_candidates_in_one_part_of_the_row(ctx, large, of):  # noqa: F811
    """The largest values are all among the first of 8 parts of 16384: more than one of them has room for, with and without room in all."""
    rng = np.random.default_rng(large)
    x = rng.standard_normal((8, 131072)).astype(np.float32)
    for row in x:
        row[rng.permutation(of)[:large]] = 5 + rng.random(large)
    check(ctx, torch.from_numpy(x).bfloat16(), rng.random(8), [1, 1, 3, 3, 1, 10, 10, 1], [1200, 1500, 2000, 4096, 1100, 1500, 3000, 50], [1, 0.9, 1, 0.9, 0.5, 1, 0.99, 1], 0)


@pytest.mark.parametrize("rows, vocab", [(1, 131072), (8, 200003), (128, 131072), (160, 131072)])
def test_thousands_take_about_the_time_of_two_thousand(ctx, rows, vocab):  # noqa: F811
    """Twice the candidates at most, and the same passes over memory: twice the time at most.  (A search in the row itself takes three to eight times as long.)"""
    g = torch.Generator("cuda").manual_seed(1)
    x, u = torch.randn(rows, vocab, generator=g, device="cuda").mul_(2).bfloat16(), torch.rand(rows, generator=g, device="cuda")
    ctx.clear_sample(x, u)

    def time(k):
        best = float("inf")
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(20):
                ctx.clear_sample(x, u, top_k=k, top_p=0.9)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best
    few = time(2000)
    assert [k for k in (2900, 3000, 3300, 3584) if time(k) > 2 * few] == []
