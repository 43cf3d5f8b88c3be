"""A step of drafted decoding in every layer: the caches of a captured step, and trees whose nodes are the tokens of a line, which is what the line itself is in one plain call."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_clear_decoder import example  # noqa: E402, F401
from test_gpu_clear_drafted import EACH, PARENTS, VOCAB, build, cached, int32  # noqa: E402

pytestmark = pytest.mark.gpu


def test_a_captured_step_in_every_layer(example):  # noqa: F811
    """Keys and values of all layers are the eager step's, after every replay."""
    from paper_2509_09424_amd import Context
    ctx = Context(12, 36, 3, 37, 1, 1, 30)
    g = torch.Generator().manual_seed(7)
    prompt = torch.randint(0, VOCAB, (60,), generator=g).cuda()
    graphed, eager = build(example, ctx), build(example, ctx)
    each, parents = int32([0, EACH, 2 * EACH, 3 * EACH]), int32(PARENTS * 3)
    flat, uniform = torch.zeros(3 * EACH, dtype=torch.int32, device="cuda"), torch.zeros(3 * EACH, device="cuda")
    run = lambda m: m.drafted(flat, parents, each, EACH, uniform, temperature=0.9, top_k=3)  # noqa: E731

    def start(m):
        for layer in m.layers:
            for x in layer.cache.tensors:
                x.zero_()
        m.lengths.zero_()
        m(m.embeddings[prompt], int32([0, 20, 40, 60]), 20)
    start(graphed)
    run(graphed)
    start(graphed)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(graphed)
    start(graphed)
    start(eager)
    for _ in range(4):
        flat.copy_(torch.randint(0, VOCAB, (3 * EACH,), generator=g))
        uniform.copy_(torch.rand(3 * EACH, generator=g))
        # the first drafts are what the roots sample, so that tokens move in every layer
        state = [[x.clone() for x in layer.cache.tensors] for layer in eager.layers], eager.lengths.clone()
        run(eager)
        flat.view(3, EACH)[:, 3] = eager.sampled.view(3, EACH)[:, 0]
        for layer, tensors in zip(eager.layers, state[0]):
            for x, y in zip(layer.cache.tensors, tensors):
                x.copy_(y)
        eager.lengths.copy_(state[1])
        _, count, _ = run(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert min(count.tolist()) >= 2 and torch.equal(graphed.lengths, eager.lengths) and torch.equal(graphed.hidden, eager.hidden)
        for layer in range(2):
            for i in range(3):
                n = int(eager.lengths[i])
                assert all(torch.equal(x, y) for x, y in zip(cached(graphed, layer, i, n), cached(eager, layer, i, n))), (layer, i)
            graphed.layers[layer].cache.check()
            eager.layers[layer].cache.check()
        assert not torch.equal(cached(eager, 0, 0, 20)[0], cached(eager, 1, 0, 20)[0])  # (the layers' are not each other's)
    graphed.free()
    eager.free()
    ctx.close()


def test_twins_of_a_line(example):  # noqa: F811
    """Tokens a, b, c behind short prompts, once as a line and once as a tree with two of b and of c, each c behind its own b: every node is what the line's token is, and so is what is
    kept of them in the caches (the twins leave the blocks' largest values alone, and the first layer's keys and values hang on token and position only: equal).  Sums in another order may
    round otherwise here and there, so the second layer and the outputs are near; trees with one wrong parent show how near that has to be: an eighth of what one wrong parent makes."""
    from paper_2509_09424_amd import Context
    ctx = Context(12, 36, 3, 37, 1, 1, 30)
    g = torch.Generator().manual_seed(12)
    lengths, right = [3, 0, 18], [-1, 0, 0, 1, 2]
    prompt = torch.randint(0, VOCAB, (21,), generator=g).cuda()
    line = torch.randint(0, VOCAB, (3, 3), generator=g)

    def run(parents):
        m = build(example, ctx)
        m(m.embeddings[prompt], int32([0, 3, 3, 21]), 18)
        which = [0, 1, 2] if parents is None else [0, 1, 1, 2, 2]
        n = len(which)
        out = m(m.embeddings[line[:, which].reshape(-1).cuda()], int32([0, n, 2 * n, 3 * n]), n, parents=parents and int32(parents * 3)).view(3, n, -1).double()
        if parents:
            ctx.clear_keep([layer.cache for layer in m.layers], m.table, int32([0, n, 2 * n, 3 * n]), m.lengths, int32([[0, 2, 4, -1, -1]] * 3), int32([3] * 3))
        kept = [[cached(m, layer, i, lengths[i] + 3) for i in range(3)] for layer in range(2)]
        for layer in m.layers:
            layer.cache.check()
        m.free()
        return out, kept
    want, want_kept = run(None)
    want = want[:, [0, 1, 1, 2, 2]]
    off = lambda got: (got - want).norm(dim=2) / want.norm(dim=2)  # noqa: E731
    apart = lambda kept, i: max(float((a - b).norm() / b.norm()) for a, b in zip(kept[1][i], want_kept[1][i]))  # noqa: E731
    got, kept = run(right)
    for i in range(3):
        assert all(torch.equal(a, b) for a, b in zip(kept[0][i], want_kept[0][i]))
    near = off(got)
    for node, parent in ((3, 0), (4, 0), (1, -1), (2, -1), (2, 1)):
        wrong = list(right)
        wrong[node] = parent
        other, other_kept = run(wrong)
        assert (off(other)[:, node] > 0.05).all() and (8 * near <= off(other)[:, node:node + 1]).all(), (node, parent)
        if node in (2, 4):  # of the path that is kept
            assert all(8 * apart(kept, i) <= apart(other_kept, i) for i in range(3))
            assert all(not torch.equal(other_kept[0][i][0], want_kept[0][i][0]) for i in range(3))  # keys of the first layer: the position
    ctx.close()
