"""The clear operators together, as the example's decoder uses them."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "clear_decoder.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("clear_decoder", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def build(example, ctx):
    return example.Decoder(ctx, layers=1, width=256, hidden=640, q_heads=4, kv_heads=2, dim=64, seqs=2, length=96, page=16, seed=3)


def test_prompts_at_once_and_token_by_token(example):
    """Two sequences of 40 and 23 tokens, all at once, in two parts, and by graph replays one by one.  The attention's results differ by the cache's roundings only:
    e4m3 rounds a value by 2^-4 of it at most, once more where a later token of its block brought a larger scale, in either of the two runs."""
    from paper_2509_09424_amd import Context
    ctx = Context(12, 36, 3, 37, 1, 1, 30)
    g = torch.Generator()
    g.manual_seed(1)
    x = [torch.randn(n, 256, generator=g).bfloat16().cuda() for n in (40, 23)]
    offsets = lambda a, b: torch.tensor([0, a, a + b], dtype=torch.int32, device="cuda")  # noqa: E731

    whole = build(example, ctx)
    out = whole(torch.cat(x), offsets(40, 23), 40)
    attention = whole.layers[0].attention.clone()
    again = build(example, ctx)
    assert torch.equal(again(torch.cat(x), offsets(40, 23), 40), out) and out.isfinite().all()  # nothing depends on an order of arrival
    again.free()

    parts = build(example, ctx)
    parts(torch.cat([x[0][:17], x[1][:23]]), offsets(17, 23), 23)
    parts(x[0][17:], offsets(23, 0), 23)
    late = parts.layers[0].attention
    near = lambda a, b: (a.double() - b.double()).norm() <= 4 * 2.0 ** -4 * b.double().norm()  # noqa: E731
    assert near(late, attention[17:40])
    parts.layers[0].cache.check()

    single = build(example, ctx)
    both = torch.empty(2, 256, dtype=torch.bfloat16, device="cuda")
    begin = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    single(both.zero_(), begin, 1)
    single.lengths.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        single(both, begin, 1)
    single.lengths.zero_()
    for t in range(23):
        both.copy_(torch.stack([x[0][t], x[1][t]]))
        graph.replay()
        torch.cuda.synchronize()
        got = single.layers[0].attention
        assert near(got[0], attention[t]) and near(got[1], attention[40 + t]), t
    single.layers[0].cache.check()
    assert single.lengths.tolist() == [23, 23]
    for m in (whole, parts, single):
        m.free()
    ctx.close()
