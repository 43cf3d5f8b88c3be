"""A step of drafted decoding as the example's decoder makes it: trees appended and attended over, a token sampled at every node, the path that agrees kept in all layers."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_clear_decoder import example  # noqa: E402, F401

pytestmark = pytest.mark.gpu

VOCAB, EACH = 300, 7
PARENTS = [-1, 0, 1, 0, 3, 4, 3]


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def build(example, ctx):  # noqa: F811
    return example.Decoder(ctx, layers=2, width=256, hidden=640, q_heads=4, kv_heads=2, dim=64, seqs=3, length=120, page=16, seed=3, vocab=VOCAB)


def cached(model, layer, i, n):
    """Keys and values of sequence i's first n tokens, as numbers."""
    k, v, ks, vs = model.layers[layer].cache.tensors
    p = torch.arange(n, device="cuda")
    page = model.table[i][p // 16].long()
    return [c[page, :, p % 16].view(torch.float8_e4m3fn).float() * s[page, :, p % 16 // 16][..., None] for c, s in ((k, ks), (v, vs))]


def near(a, b):
    """By the cache's roundings: e4m3 rounds a value by 2^-4 of it at most, again where a token that came later, kept or not, brought a larger scale, in either of the two runs."""
    return (a.double() - b.double()).norm() <= 4 * 2.0 ** -4 * b.double().norm()


def test_steps_against_one_token_at_a_time(example):  # noqa: F811
    """Sequences of 40, 16 and 21 tokens, three steps: node by node near to the same tokens decoded alone; what is kept is what was decoded."""
    from paper_2509_09424_amd import Context
    ctx = Context(12, 36, 3, 37, 1, 1, 30)
    g = torch.Generator().manual_seed(5)
    lengths = [40, 16, 21]
    prompt = torch.randint(0, VOCAB, (sum(lengths),), generator=g).cuda()
    begin = int32([0, 40, 56, 77])
    trees, alone = build(example, ctx), build(example, ctx)
    for m in (trees, alone):
        m(m.embeddings[prompt], begin, 40)
    last = [int(prompt[39]), int(prompt[55]), int(prompt[76])]
    each = int32([0, EACH, 2 * EACH, 3 * EACH])
    parents = int32(PARENTS * 3)
    kept = list(lengths)
    for step in range(3):
        tokens = torch.randint(0, VOCAB, (3, EACH), generator=g)
        tokens[:, 0] = torch.tensor(last)
        # the random numbers that make token 3 and 4 (5 in the last step) of the first sequence, token 1 of the second, and nothing of the third agree
        uniform, flat = torch.rand(3 * EACH, generator=g).cuda(), tokens.view(-1).int().cuda()
        before = trees.lengths.clone()
        # greedy samples first, to draft some of them
        probe = build(example, ctx)
        for a, b in zip(probe.layers, trees.layers):
            for x, y in zip(a.cache.tensors, b.cache.tensors):
                x.copy_(y)
        probe.lengths.copy_(before)
        for _ in range(3):  # a child's sample follows its parent's
            probe.lengths.copy_(before)
            probe.drafted(flat, parents, each, EACH, uniform, temperature=0)
            s = probe.sampled.view(3, EACH)
            flat.view(3, EACH)[0, 3], flat.view(3, EACH)[0, 4], flat.view(3, EACH)[1, 1] = s[0, 0], s[0, 3], s[1, 0]
            if step == 2:
                flat.view(3, EACH)[0, 5] = s[0, 4]
            for a, b in zip(probe.layers, trees.layers):
                for x, y in zip(a.cache.tensors, b.cache.tensors):
                    x.copy_(y)
        probe.free()
        tokens = flat.view(3, EACH).tolist()
        path, count, following = trees.drafted(flat, parents, each, EACH, uniform, temperature=0)
        hidden, sampled = trees.hidden.view(3, EACH, -1).clone(), trees.sampled.view(3, EACH).tolist()
        # the path follows from what was sampled
        for i in range(3):
            line = [0]
            while True:
                child = next((c for c in range(line[-1] + 1, EACH) if PARENTS[c] == line[-1] and tokens[i][c] == sampled[i][line[-1]]), None)
                if child is None:
                    break
                line.append(child)
            assert path[i].tolist() == line + [-1] * (EACH - len(line)) and int(count[i]) == len(line) and int(following[i]) == sampled[i][line[-1]]
            kept[i] += len(line)
        assert trees.lengths.tolist() == kept and (trees.lengths - before).tolist() == count.tolist() and int(count[0]) >= 3
        # the kept tokens decoded one by one
        for j in range(int(count.max())):
            new = [int(j < int(c)) for c in count]
            x = [alone.embeddings[tokens[i][int(path[i][j])]] for i in range(3) if new[i]]
            offsets = int32([0, new[0], new[0] + new[1], sum(new)])
            out = alone(torch.stack(x), offsets, 1)
            got = torch.stack([hidden[i][int(path[i][j])] for i in range(3) if new[i]])
            assert near(got, out), (step, j)
        assert alone.lengths.tolist() == kept
        for layer in range(2):
            for i in range(3):
                for a, b in zip(cached(trees, layer, i, kept[i]), cached(alone, layer, i, kept[i])):
                    assert near(a, b), (step, layer, i)
        last = following.tolist()
    for m in (trees, alone):
        for layer in m.layers:
            layer.cache.check()
        m.free()
    ctx.close()


def test_a_captured_step_and_forks(example):  # noqa: F811
    """The step as a graph, replayed with other drafts and random numbers, is the step itself; forked sequences then go on as their source would."""
    from paper_2509_09424_amd import Context
    ctx = Context(12, 36, 3, 37, 1, 1, 30)
    g = torch.Generator().manual_seed(6)
    prompt = torch.randint(0, VOCAB, (60,), generator=g).cuda()
    graphed, eager = build(example, ctx), build(example, ctx)
    each, parents = int32([0, EACH, 2 * EACH, 3 * EACH]), int32(PARENTS * 3)
    flat, uniform = torch.empty(3 * EACH, dtype=torch.int32, device="cuda"), torch.empty(3 * EACH, device="cuda")
    run = lambda m: m.drafted(flat, parents, each, EACH, uniform, temperature=0.9, top_k=20, top_p=0.9, min_p=0.01)  # noqa: E731

    def start(m):
        for layer in m.layers:
            for x in layer.cache.tensors:
                x.zero_()
        m.lengths.zero_()
        m(m.embeddings[prompt], int32([0, 20, 40, 60]), 20)
    fill = lambda: (flat.copy_(torch.randint(0, 6, (3 * EACH,), generator=g)), uniform.copy_(torch.rand(3 * EACH, generator=g)))  # noqa: E731
    start(graphed)
    fill()
    run(graphed)
    start(graphed)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        path, count, following = run(graphed)
    start(graphed)
    start(eager)
    for _ in range(4):
        fill()
        graph.replay()
        want = run(eager)
        torch.cuda.synchronize()
        assert torch.equal(path, want[0]) and torch.equal(count, want[1]) and torch.equal(following, want[2]) and torch.equal(graphed.lengths, eager.lengths)
        assert torch.equal(graphed.hidden, eager.hidden)
        for a, b in zip(graphed.layers, eager.layers):
            for i in range(3):
                n = int(eager.lengths[i])
                assert all(torch.equal(x, y) for x, y in zip(cached(graphed, 0, i, n), cached(eager, 0, i, n)))
            a.cache.check()
            b.cache.check()
    # all three go on as the second did: on its own pages, and on those that the others had
    source, n = eager.lengths.tolist()[1], eager.lengths.tolist()[1] // 16
    wide = eager.table.clone()
    eager.fork(int32([1, 1, 1]), int32([int(wide[0, n]), int(wide[1, n]), int(wide[2, n])]))
    assert eager.lengths.tolist() == [source] * 3
    for i in range(3):
        eager.table[i, n + 1:] = wide[i, n + 1:]
    flat.copy_(torch.randint(0, VOCAB, (EACH,), generator=g).repeat(3))
    uniform.copy_(torch.rand(EACH, generator=g).repeat(3))
    path, count, following = run(eager)
    assert torch.equal(eager.hidden.view(3, EACH, -1)[0], eager.hidden.view(3, EACH, -1)[1]) and torch.equal(eager.hidden.view(3, EACH, -1)[0], eager.hidden.view(3, EACH, -1)[2])
    assert count.tolist() == [int(count[0])] * 3 and following.tolist() == [int(following[0])] * 3
    for layer in eager.layers:
        layer.cache.check()
    graphed.free()
    eager.free()
    ctx.close()
