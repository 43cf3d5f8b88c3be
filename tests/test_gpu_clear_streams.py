"""The clear calls on a stream that is given: what they make belongs to it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_clear import Cache, ctx  # noqa: E402, F401

TOKENS = 3


def calls(ctx, c):
    """(name, size in bytes of a tensor that the call makes, call): every call whose output the binding makes."""
    x, gain = torch.randn(TOKENS, 4096, device="cuda"), torch.ones(4096, device="cuda")
    codes, scales = torch.ones(TOKENS, 4096, dtype=torch.int8, device="cuda"), torch.ones(TOKENS, device="cuda")
    weights = ctx.clear_weights_prepare(np.ones((4096, 512), dtype=np.int8), np.ones(512, dtype=np.float32))
    cache = c.wrap(ctx)
    q, k = torch.randn(TOKENS, 8, 64, device="cuda").bfloat16(), torch.randn(TOKENS, 1, 64, device="cuda").bfloat16()
    v, cos = k.clone(), torch.ones(64, 32, device="cuda")
    return [("norm", TOKENS * 4096, lambda s: ctx.clear_norm(x, gain, stream=s)[0]), ("norm's scales", 4 * TOKENS, lambda s: ctx.clear_norm(x, gain, codes=codes, stream=s)[1]),
            ("product", 2 * TOKENS * 512, lambda s: ctx.clear_matmul(weights, codes, scales, dtype=torch.bfloat16, stream=s)),
            ("append", 2 * TOKENS * 512, lambda s: ctx.clear_append(cache, *c.where, k, v, cos, cos, q=q, stream=s)),
            ("attention", 2 * TOKENS * 512, lambda s: ctx.clear_attention(cache, *c.where, q, stream=s))]


def test_outputs_come_from_the_stream_that_writes_them(ctx):
    """A block that the current stream has freed, of just the size: its earlier work may still be under way, so a call on another stream may not get it."""
    c = Cache(ctx, [20, 5], [2, 1], 1, 64, 16, 1)
    c.fill_new()
    side = torch.cuda.Stream()
    for name, size, call in calls(ctx, c):
        want = call(None)
        torch.cuda.synchronize()
        blocks = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(8)]
        freed = {b.data_ptr() for b in blocks}
        del blocks
        got = [call(side.cuda_stream) for _ in range(4)]
        assert not freed & {g.data_ptr() for g in got}, name
        torch.cuda.synchronize()
        assert all(torch.equal(g, want) for g in got), name
        # and the other way round: what a call of the side stream has left there serves its next one, and a call that is given the current stream is like any other
        mine = {g.data_ptr() for g in got}
        del got
        assert call(side.cuda_stream).data_ptr() in mine, name
        with torch.cuda.stream(side):
            assert torch.equal(call(side.cuda_stream), call(None)), name
            on_default = call(torch.cuda.default_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(on_default, want) and on_default.data_ptr() not in mine, name
