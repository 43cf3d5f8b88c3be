"""The example's decoder, call by call: what every clear call of it is given and gives, against the definitions in 64 bits, and a captured step against the same step
without a graph, bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_clear import U32, Cache, append_reference, ctx, half_step, norm_reference, same_codes  # noqa: E402, F401
from test_gpu_clear_attention_bounds import check  # noqa: E402
from test_gpu_clear_decoder import build, example  # noqa: E402, F401


class Watched:
    """A context whose clear calls are compared with their definitions as they are made."""

    def __init__(self, ctx):
        self.ctx, self.W, self.counts = ctx, {}, {}

    def __getattr__(self, name):
        return getattr(self.ctx, name)

    def clear_weights_prepare(self, W, w_scales, group=0):
        handle = self.ctx.clear_weights_prepare(W, w_scales, group)
        self.W[handle] = torch.from_numpy(W).double(), torch.from_numpy(w_scales).double()
        return handle

    def count(self, name):
        self.counts[name] = self.counts.get(name, 0) + 1

    def clear_norm(self, x, gain, residual=None, sum_out=None):
        h, codes, scales, _ = norm_reference(x.cpu(), gain.cpu(), None if residual is None else residual.cpu(), 1e-5)
        got = self.ctx.clear_norm(x, gain, residual=residual, sum_out=sum_out)
        assert np.array_equal(got[0].cpu().numpy(), codes)
        assert ((got[1].cpu().double() - scales).abs() <= 64 * U32 * scales).all()  # as in test_norm
        assert sum_out is None or torch.equal(sum_out.cpu(), h)
        self.count("norm")
        return got

    def clear_matmul(self, weights, codes, scales, dtype):
        got = self.ctx.clear_matmul(weights, codes, scales, dtype=dtype)
        W, w_scales = self.W[weights]
        want = codes.cpu().double() @ W * w_scales * scales.cpu().double()[:, None]
        assert ((got.cpu().double() - want).abs() <= (half_step("bf16") * (1 + 1e-6) + 3 * U32) * want.abs()).all()  # a whole number times two scales, rounded once
        self.count("matmul")
        return got

    def state(self, cache, table, begin, lengths):
        c = Cache.__new__(Cache)
        c.table, c.begin = table.cpu(), begin.cpu()
        c.ctxs, c.news = lengths.tolist(), (begin[1:] - begin[:-1]).tolist()
        c.heads, c.dim, c.page, c.tokens = cache.heads, cache.dim, cache.page, int(begin[-1])
        parts = [t.cpu().clone() for t in cache.tensors]
        c.codes, c.scales = dict(zip("kv", parts[:2])), dict(zip("kv", parts[2:]))
        return c

    def clear_append(self, cache, table, begin, lengths, k, v, cos, sin, q=None, q_out=None, max_new=None):
        before = self.state(cache, table, begin, lengths)
        codes, scales = append_reference(before, k.cpu(), v.cpu(), cos.cpu().numpy(), sin.cpu().numpy(), cache.dim, "half")
        out = self.ctx.clear_append(cache, table, begin, lengths, k, v, cos, sin, q=q, q_out=q_out, max_new=max_new)
        after = self.state(cache, table, begin, lengths)
        for x in "kv":
            assert same_codes(after.codes[x], codes[x]) and torch.equal(after.scales[x], scales[x])
        self.count("append")
        return out

    def clear_attention(self, cache, table, begin, lengths, q, max_new=None, max_length=None):
        got = self.ctx.clear_attention(cache, table, begin, lengths, q, max_new=max_new, max_length=max_length)
        check(self.state(cache, table, begin, lengths), "bf16", got, q.cpu())
        self.count("attention")
        return got


def test_every_call_of_prompts_and_of_single_tokens(example, ctx):
    """Two sequences of 40 and 23 tokens at once, then in two parts, then token by token."""
    g = torch.Generator()
    g.manual_seed(1)
    x = [torch.randn(n, 256, generator=g).bfloat16().cuda() for n in (40, 23)]
    offsets = lambda a, b: torch.tensor([0, a, a + b], dtype=torch.int32, device="cuda")  # noqa: E731
    watched = Watched(ctx)
    whole = build(example, watched)
    assert whole(torch.cat(x), offsets(40, 23), 40).isfinite().all()
    parts = build(example, watched)
    parts(torch.cat([x[0][:17], x[1]]), offsets(17, 23), 23)
    parts(x[0][17:], offsets(23, 0), 23)
    single = build(example, watched)
    for t in range(23):
        single(torch.stack([x[0][t], x[1][t]]), offsets(1, 1), 1)
    assert watched.counts == {"norm": 26 * 4, "matmul": 26 * 4, "append": 26, "attention": 26}
    for m in (whole, parts, single):
        m.layers[0].cache.check()
        m.free()


def test_a_captured_step_is_the_step(example, ctx):
    g = torch.Generator()
    g.manual_seed(2)
    x = torch.randn(30, 2, 256, generator=g).bfloat16().cuda()
    begin = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    eager, captured = build(example, ctx), build(example, ctx)
    both = torch.zeros(2, 256, dtype=torch.bfloat16, device="cuda")
    captured(both, begin, 1)
    captured.lengths.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = captured(both, begin, 1)
    captured.lengths.zero_()
    for t in range(30):
        want = eager(x[t], begin, 1)
        both.copy_(x[t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(captured.layers[0].attention, eager.layers[0].attention), t
    for m in (eager, captured):
        m.layers[0].cache.check()
        m.free()
