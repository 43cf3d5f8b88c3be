"""The calls of drafted decoding on other streams, in graphs that share the workspace, and on pages past 32 bits."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_clear import Cache, ctx  # noqa: E402, F401
from test_gpu_clear_tree import trees  # noqa: E402

pytestmark = pytest.mark.gpu


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def calls(ctx, c, cache, g):  # noqa: F811
    """(name, call) of every call that returns something."""
    x, u = torch.randn(3, 40000, generator=g).cuda(), torch.rand(3, generator=g).cuda()
    tokens = c.tokens
    parents, drafted, sampled = trees(c.news, 1).cuda(), int32([i % 3 for i in range(tokens)]), int32([(i + 1) % 3 for i in range(tokens)])
    q, k = torch.randn(tokens, 4, 64, generator=g).bfloat16().cuda(), torch.randn(tokens, 1, 64, generator=g).bfloat16().cuda()
    return [("sample", lambda s=None: ctx.clear_sample(x, u, top_p=0.9, stream=s)), ("sample of candidates", lambda s=None: ctx.clear_sample(x, u, top_k=40, stream=s)),
            ("append", lambda s=None: ctx.clear_append(cache, *c.where, k, k, None, None, q=q, parents=parents, stream=s)),
            ("attention", lambda s=None: ctx.clear_attention(cache, *c.where, q, parents=parents, stream=s)),
            ("accept", lambda s=None: torch.cat([t.flatten() for t in ctx.clear_accept(c.where[1], parents, drafted, sampled, stream=s)])),
            ("fork", lambda s=None: torch.cat([t.flatten() for t in ctx.clear_fork(cache, c.where[0], c.where[2], int32([0]), int32([int(c.table[0, c.ctxs[0] // c.page])]), stream=s)]))]


def test_a_stream_that_is_given(ctx):  # noqa: F811
    g = torch.Generator().manual_seed(1)
    c = Cache(ctx, [2000, 5], [9, 4], 1, 64, 16, 1)
    c.fill_new()
    cache = c.wrap(ctx)
    side = torch.cuda.Stream()
    for name, call in calls(ctx, c, cache, g):
        want = call()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            got = call()
        side.synchronize()
        assert torch.equal(got, want), name
        torch.cuda.synchronize()
        if name not in ("accept", "fork"):  # (their parts are joined above on the current stream)
            got = call(side.cuda_stream)
            torch.cuda.synchronize()
            assert torch.equal(got, want), name
    cache.check()
    cache.free()


def test_graphs_that_share_the_workspace(ctx):  # noqa: F811
    """A graph of split sampling and one of split attention, replayed in turn with eager calls between."""
    g = torch.Generator().manual_seed(2)
    c = Cache(ctx, [3000, 700], [9, 30], 1, 64, 16, 2)
    c.fill_new()
    cache = c.wrap(ctx)
    made = [call for name, call in calls(ctx, c, cache, g) if name in ("sample", "sample of candidates", "attention")]
    want = [call() for call in made]
    graphs = []
    for call in made:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for order in ((0, 1, 2), (2, 0, 1), (1, 2, 0)):
        for i in order:
            graphs[i][1].zero_()
            graphs[i][0].replay()
            torch.cuda.synchronize()
            assert torch.equal(graphs[i][1], want[i])
            assert torch.equal(made[(i + 1) % 3](), want[(i + 1) % 3])
    cache.free()


def test_a_first_call_that_is_captured():
    """A context without a cache or weights has no workspace to split rows with, and makes none within a capture: the tokens are the same."""
    from paper_2509_09424_amd import Context
    g = torch.Generator().manual_seed(3)
    x, u = torch.randn(4, 100000, generator=g).cuda(), torch.rand(4, generator=g).cuda()
    out = torch.empty(4, dtype=torch.int32, device="cuda")
    fresh, other = Context(12, 36, 3, 37, 1, 1, 30), Context(12, 36, 3, 37, 1, 1, 30)
    for settings in (dict(top_p=0.9), dict(top_k=700, top_p=0.8), dict(min_p=0.01), dict(temperature=0), dict(top_k=5000)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fresh.clear_sample(x, u, out=out, **settings)
        for _ in range(2):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, other.clear_sample(x, u, **settings)), settings
    fresh.close()
    other.close()


def test_pages_past_32_bits(ctx):  # noqa: F811
    """The same sequences on pages at the end of arrays of 4.3 GiB each."""
    c = Cache(ctx, [100, 37], [9, 20], 8, 128, 64, 7)
    c.fill_new()
    pages = c.codes["k"].shape[0]
    far = (1 << 16) + 500  # 64 KiB a page
    near = c.wrap(ctx)
    big = [torch.empty(far + pages + 1, 8, 64, 128, dtype=torch.uint8, device="cuda") for _ in "kv"] + [torch.empty(far + pages + 1, 8, 4, device="cuda") for _ in "kv"]
    for t, small in zip(big, c.dev):
        t[far:far + pages] = small
    cache = ctx.clear_cache(*big)
    g = torch.Generator().manual_seed(8)
    q, k = torch.randn(29, 16, 128, generator=g).bfloat16().cuda(), torch.randn(29, 8, 128, generator=g).bfloat16().cuda()
    parents = trees(c.news, 4).cuda()
    table = torch.where(c.where[0] >= 0, c.where[0] + far, -1)
    path, count = int32([[0, 3, 8] + [-1] * 17, [0, 1, 5, 19] + [-1] * 16]), int32([3, 4])
    for at, one in ((near, c.where[0]), (cache, table)):
        ctx.clear_append(at, one, *c.where[1:], k, k, None, None, parents=parents, max_new=20)
    assert torch.equal(ctx.clear_attention(near, *c.where, q, parents=parents, max_new=20), ctx.clear_attention(cache, table, *c.where[1:], q, parents=parents, max_new=20))
    for at, one in ((near, c.where[0]), (cache, table)):
        ctx.clear_keep(at, one, *c.where[1:], path, count)
    for t, small in zip(big, c.dev):
        assert torch.equal(t[far:far + pages].view(torch.uint8), small.view(torch.uint8))
    _, lengths = ctx.clear_fork(cache, table, c.where[2], int32([0]), int32([far + pages]))
    used = int(table[0, 1])
    assert lengths.tolist() == [100] and all(torch.equal(t[far + pages, :, :48], t[used, :, :48]) for t in big[:2]) and all(torch.equal(t[far + pages, :, :3], t[used, :, :3]) for t in big[2:])
    near.check()
    cache.check()
    near.free()
    cache.free()
