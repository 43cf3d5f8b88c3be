"""A ternary decoder on clear activations: the layer that the library computes on ciphertexts, for requests that are not encrypted.

    python examples/clear_decoder.py [--layers 4] [--prompt 512] [--steps 32] [--draft]

One layer is norm -> queries, keys and values (one ternary product) -> rotation and append to the paged 8-bit cache -> attention -> norm -> output
projection -> norm with the residual's addition -> up projection -> norm of the squared positive part -> down projection.  Weights are random;
a decoding step is captured into a graph once and replayed for every token, with lengths advanced on the device.

With --draft, a step takes a tree of drafted tokens for every sequence: they are embedded, appended and attended over, a token is sampled at each of them, the path that agrees is
kept in the caches of all layers, and what was sampled at its end begins the next tree.  That step is a graph too; nothing of it is decided on the host.
"""
import argparse
import os
import sys
import time

import numpy as np

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import torch  # noqa: E402

from paper_2509_09424_amd import Context  # noqa: E402


class Layer:
    def __init__(self, ctx, rng, width, hidden, q_heads, kv_heads, dim, pages, page):
        self.ctx, self.q_heads, self.kv_heads, self.dim, self.width = ctx, q_heads, kv_heads, dim, width
        heads = q_heads + 2 * kv_heads

        def ternary(d, m):  # values of unit size keep theirs: 0.6 d of the weights are not zero
            return ctx.clear_weights_prepare(rng.choice(np.array([-1, 0, 1], dtype=np.int8), size=(d, m), p=[0.3, 0.4, 0.3]), np.full(m, (0.6 * d) ** -0.5, dtype=np.float32))

        self.qkv, self.out, self.up, self.down = ternary(width, heads * dim), ternary(q_heads * dim, width), ternary(width, hidden), ternary(hidden, width)
        self.gains = [torch.ones(n, dtype=torch.bfloat16, device="cuda") for n in (width, q_heads * dim, width, hidden)]
        cache = [torch.zeros(pages, kv_heads, page, dim, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = [torch.zeros(pages, kv_heads, page // 16, device="cuda") for _ in range(2)]
        self.cache = ctx.clear_cache(*cache, *scales)

    def __call__(self, x, residual, seqs, turn, tree={}, **bounds):
        """(what the layer adds, the sum before it): both enter the next layer's first norm."""
        ctx, q = self.ctx, self.q_heads
        codes, scales = ctx.clear_norm(x, self.gains[0], residual=residual, sum_out=residual)
        heads = ctx.clear_matmul(self.qkv, codes, scales, dtype=x.dtype).view(x.shape[0], -1, self.dim)
        queries = ctx.clear_append(self.cache, *seqs, heads[:, q:q + self.kv_heads], heads[:, q + self.kv_heads:], *turn, q=heads[:, :q], q_out=heads[:, :q], max_new=bounds["max_new"], **tree)
        self.attention = ctx.clear_attention(self.cache, *seqs, queries, **bounds, **tree).view(x.shape[0], -1)
        y = ctx.clear_matmul(self.out, *ctx.clear_norm(self.attention, self.gains[1]), dtype=x.dtype)
        codes, scales = ctx.clear_norm(y, self.gains[2], residual=residual, sum_out=residual)
        hidden = ctx.clear_matmul(self.up, codes, scales, dtype=x.dtype).relu_().square_()
        return ctx.clear_matmul(self.down, *ctx.clear_norm(hidden, self.gains[3]), dtype=x.dtype), residual

    def free(self):
        for h in (self.qkv, self.out, self.up, self.down, self.cache):
            h.free()


class Decoder:
    """`seqs` sequences of up to `length` tokens through `layers` layers; embeddings in, the last layer's sums out.  With a vocabulary, tokens in and tokens out (drafted)."""

    def __init__(self, ctx, layers=2, width=2560, hidden=6912, q_heads=20, kv_heads=5, dim=128, seqs=4, length=2048, page=64, seed=0, vocab=0):
        rng = np.random.default_rng(seed)
        width_pages = -(-length // page)
        self.layers = [Layer(ctx, rng, width, hidden, q_heads, kv_heads, dim, seqs * width_pages, page) for _ in range(layers)]
        order = rng.permutation(seqs * width_pages).astype(np.int32).reshape(seqs, width_pages)
        self.table = torch.from_numpy(order).cuda()
        self.lengths = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        angle = np.arange(length)[:, None] * 10000.0 ** (-np.arange(0, dim, 2) / dim)
        self.turn = torch.from_numpy(np.cos(angle).astype(np.float32)).cuda(), torch.from_numpy(np.sin(angle).astype(np.float32)).cuda()
        self.length, self.width, self.ctx, self.head = length, width, ctx, None
        if vocab:
            self.embeddings = torch.from_numpy(rng.standard_normal((vocab, width), dtype=np.float32)).cuda().bfloat16()
            self.head = ctx.clear_weights_prepare(rng.choice(np.array([-1, 0, 1], dtype=np.int8), size=(width, vocab), p=[0.3, 0.4, 0.3]), np.full(vocab, 3 * (0.6 * width) ** -0.5, dtype=np.float32))
            self.gain = torch.ones(width, dtype=torch.bfloat16, device="cuda")

    def __call__(self, x, begin, max_new, max_length=None, parents=None):
        """x: [tokens][width] embeddings of the new tokens, sequence i's from begin[i] on.  Advances the lengths, unless the tokens are trees (parents)."""
        seqs, residual, tree = (self.table, begin, self.lengths), torch.zeros_like(x), {} if parents is None else {"parents": parents}
        for layer in self.layers:
            x, residual = layer(x, residual, seqs, self.turn, tree, max_new=max_new, max_length=max_length or self.length)
        if parents is None:
            self.lengths += begin[1:] - begin[:-1]
        return x + residual

    def drafted(self, tokens, parents, begin, max_new, uniform, **settings):
        """A step with trees of drafted tokens (int32 [tokens]; the first of each sequence is its last one).  Advances the lengths by what is kept; returns (path, count, following)."""
        ctx = self.ctx
        self.hidden = self(self.embeddings[tokens.long()], begin, max_new, parents=parents)
        logits = ctx.clear_matmul(self.head, *ctx.clear_norm(self.hidden, self.gain), dtype=torch.bfloat16)
        self.sampled = ctx.clear_sample(logits, uniform, **settings)
        path, count, following = ctx.clear_accept(begin, parents, tokens, self.sampled, max_new=max_new)
        ctx.clear_keep([layer.cache for layer in self.layers], self.table, begin, self.lengths, path, count)
        self.lengths += count
        return path, count, following

    def fork(self, source, fresh):
        """Sequence i goes on as source[i] did; the page that it had begun is copied to page fresh[i]."""
        self.table, self.lengths = self.ctx.clear_fork([layer.cache for layer in self.layers], self.table, self.lengths, source, fresh)

    def free(self):
        for layer in self.layers:
            layer.free()
        if self.head:
            self.head.free()


def drafts(model, following, fan, generator):
    """Trees of 1 + 2 fan tokens: the last token, `fan` drafts of the next one, one more behind each of them.  (Random ones: a program would ask a smaller model.)"""
    seqs = following.shape[0]
    tokens = torch.randint(0, model.embeddings.shape[0], (seqs, 1 + 2 * fan), generator=generator, device="cuda", dtype=torch.int32)
    tokens[:, 0] = following
    parents = torch.tensor([-1] + [0] * fan + list(range(1, 1 + fan)), dtype=torch.int32, device="cuda").repeat(seqs)
    return tokens.view(-1), parents


def draft(a, ctx):
    fan, vocab = 3, 32000
    each = 1 + 2 * fan
    model = Decoder(ctx, layers=a.layers, seqs=a.seqs, length=a.prompt + 3 * (a.steps + 8) + each, vocab=vocab)
    begin = torch.arange(a.seqs + 1, dtype=torch.int32, device="cuda")
    prompt = torch.randint(0, vocab, (a.seqs, a.prompt), device="cuda")
    rest = a.prompt - 1  # a prompt's last token is the first of a tree
    if rest:
        model(model.embeddings[prompt[:, :rest].reshape(-1)], begin * rest, rest, rest)
    generator = torch.Generator(device="cuda")
    tokens, parents = drafts(model, prompt[:, rest].int(), fan, generator)
    uniform, total = torch.rand(a.seqs * each, device="cuda"), torch.zeros(a.seqs, dtype=torch.int32, device="cuda")

    def step():
        _, count, following = model.drafted(tokens, parents, begin * each, each, uniform, temperature=0.8, top_k=50, top_p=0.95)
        total.add_(count)
        tokens.view(a.seqs, each)[:, 0] = following
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    total.zero_()
    t = time.perf_counter()
    for _ in range(a.steps):
        uniform.uniform_()
        graph.replay()
    torch.cuda.synchronize()
    print("a step of %d sequences with trees of %d tokens: %.1f us (graph), %.2f tokens kept of each" % (a.seqs, each, 1e6 * (time.perf_counter() - t) / a.steps, total.float().mean() / a.steps))
    for layer in model.layers:
        layer.cache.check()
    model.free()


def main():
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("layers", 4), ("prompt", 512), ("steps", 32), ("seqs", 4)):
        parser.add_argument("--" + name, type=int, default=value)
    parser.add_argument("--draft", action="store_true", help="trees of drafted tokens in place of one token a step")
    a = parser.parse_args()
    ctx = Context(12, 36, 3, 37, 1, 1, 30)
    if a.draft:
        draft(a, ctx)
        ctx.close()
        return
    model = Decoder(ctx, layers=a.layers, seqs=a.seqs, length=a.prompt + a.steps + 8)
    x = torch.randn(a.seqs * a.prompt, model.width, device="cuda").bfloat16()
    begin = torch.arange(a.seqs + 1, dtype=torch.int32, device="cuda") * a.prompt
    torch.cuda.synchronize()
    t = time.perf_counter()
    model(x, begin, a.prompt, a.prompt)
    torch.cuda.synchronize()
    print("prompts of %d tokens, %d sequences, %d layers: %.2f ms (first pass)" % (a.prompt, a.seqs, a.layers, 1e3 * (time.perf_counter() - t)))
    one, ones = torch.randn(a.seqs, model.width, device="cuda").bfloat16(), torch.arange(a.seqs + 1, dtype=torch.int32, device="cuda")
    step = lambda: model(one, ones, 1)  # noqa: E731
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        graph.replay()
    torch.cuda.synchronize()
    print("a decoding step of %d sequences: %.1f us (graph)" % (a.seqs, 1e6 * (time.perf_counter() - t) / a.steps))
    for layer in model.layers:
        layer.cache.check()
    assert out.isfinite().all()
    model.free()
    ctx.close()


if __name__ == "__main__":
    main()
