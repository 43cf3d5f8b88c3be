"""The accepted path of drafted tokens, moving them together in the caches of several layers, and forks of sequences, against plain loops: whole numbers, codes and scales are equal."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_clear import Cache, ctx, e4m3, same_codes  # noqa: E402, F401
from test_gpu_clear_tree import lines, trees  # noqa: E402

pytestmark = pytest.mark.gpu


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- accept -----------------------------------------------------------------------------------------------------------------


def accept_reference(news, parents, drafted, sampled, width):
    path, count, following, first = [], [], [], 0
    for n in news:
        line, node = [], 0 if n else None
        while node is not None:
            line.append(node)
            node = next((c for c in range(node + 1, n) if (parents[first + c] if parents is not None else c - 1) == node and drafted[first + c] == sampled[first + node] >= 0), None)
        path.append(line + [-1] * (width - len(line)))
        count.append(len(line))
        following.append(sampled[first + line[-1]] if n else -1)
        first += n
    return path, count, following


@pytest.mark.parametrize("news, shape", [([1], "chain"), ([64], "chain"), ([5, 0, 7, 64, 1], "mixed"), ([30, 64], "star"), ([9, 3], "roots"), ([i % 65 for i in range(200)], "mixed")])
@pytest.mark.parametrize("agree", [0.0, 0.7, 1.0])
def test_accept(ctx, news, shape, agree):  # noqa: F811
    rng = np.random.default_rng(sum(news))
    parents = trees(news, 1, shape).tolist()
    tokens = sum(news)
    drafted, sampled = rng.integers(0, 9, tokens).tolist(), rng.integers(-1, 9, tokens).tolist()  # few different ones: children of one node with the same token
    first = 0
    for n in news:
        for t in range(n):
            if parents[first + t] >= 0 and rng.random() < agree:
                sampled[first + parents[first + t]] = drafted[first + t]
        first += n
    begin = int32(np.concatenate([[0], np.cumsum(news)]))
    width = max(news)
    want = accept_reference(news, parents, drafted, sampled, width)
    path, count, following = ctx.clear_accept(begin, int32(parents), int32(drafted), int32(sampled), max_new=width)
    assert (path.tolist(), count.tolist(), following.tolist()) == want
    if shape == "chain":
        path, count, following = ctx.clear_accept(begin, None, int32(drafted), int32(sampled), max_new=width)
        assert (path.tolist(), count.tolist(), following.tolist()) == want
    # in wider arrays of the caller's, whose other places stay
    wide = torch.full((len(news), width + 3), 77, dtype=torch.int32, device="cuda")
    ctx.clear_accept(begin, int32(parents), int32(drafted), int32(sampled), path=wide[:, :width])
    assert wide[:, :width].tolist() == want[0] and (wide[:, width:] == 77).all()


def test_accept_of_numbers_that_do_not_fit(ctx):  # noqa: F811
    """Parents that are none are never a node's child; offsets that do not fit give an empty path."""
    drafted, sampled = int32([1, 2, 3, 4]), int32([2, 3, 4, 5])
    for parents in ([-1, 0, 5, -7], [-1, 0, 2 ** 31 - 1, -2 ** 31], [3, 0, 0, 3]):
        path, count, following = ctx.clear_accept(int32([0, 4]), int32(parents), drafted, sampled)
        assert path.tolist() == [[0, 1, -1, -1]] and count.tolist() == [2] and following.tolist() == [3]
    for begin in ([0, 5], [-1, 3], [3, 1], [-2 ** 31, 2 ** 31 - 1]):
        path, count, following = ctx.clear_accept(int32(begin), None, drafted, sampled)
        assert path.tolist() == [[-1] * 4] and count.tolist() == [0] and following.tolist() == [-1]
    path, count, _ = ctx.clear_accept(int32([0, 4]), None, drafted, sampled, max_new=3)
    assert path.tolist() == [[-1] * 3] and count.tolist() == [0]


# ---- keep -------------------------------------------------------------------------------------------------------------------


def keep_reference(c, paths):
    codes, scales = {x: t.clone() for x, t in c.codes.items()}, {x: t.clone() for x, t in c.scales.items()}
    place = lambda i, p: (int(c.table[i, p // c.page]), p % c.page)  # noqa: E731
    for i, (length, path) in enumerate(zip(c.ctxs, paths)):
        first = next((j for j, p in enumerate(path) if p != j), None)
        if first is None:
            continue
        for start in range((length + first) // 16 * 16, length + len(path), 16):
            holds = [(t, place(i, t if t < length + first else length + path[t - length])) for t in range(start, min(start + 16, length + len(path)))]
            one, r = place(i, start)
            for x in "kv":
                for h in range(c.heads):
                    was = [float(c.scales[x][p, h, q // 16]) for _, (p, q) in holds]
                    scales[x][one, h, r // 16] = max(was)
                    for (t, (p, q)), s in zip(holds, was):
                        code = c.codes[x][p, h, q]
                        codes[x][one, h, r + t - start] = (e4m3(code) * (s / max(was))).to(torch.float8_e4m3fn).view(torch.uint8) if s != max(was) else code
    return codes, scales


def a_path(parents, first, n, rng):
    return sorted(lines(parents, first, n)[int(rng.integers(0, n))]) if n else []


@pytest.mark.parametrize("ctxs, news, heads, dim, page", [([0], [1], 1, 64, 16), ([0, 5, 16, 33], [64, 64, 20, 0], 2, 128, 16), ([100, 250, 7], [64, 31, 64], 3, 96, 64), ([15, 31], [64, 63], 1, 256, 32),
                                                          ([1000, 3], [17, 64], 2, 192, 48), ([8] * 40, [3 + i for i in range(40)], 2, 64, 32)])
def test_keep(ctx, ctxs, news, heads, dim, page):  # noqa: F811
    rng = np.random.default_rng(dim + page)
    for shape in ("mixed", "star", "sparse"):
        layers = [Cache(ctx, ctxs, news, heads + (k == 2), dim if k < 2 else 64, page, 5) for k in range(3)]  # one table, other heads in the last
        for k, c in enumerate(layers):
            c.table = layers[0].table
            c.fill_new((-8 - k, 3))
        parents, paths = trees(news, 2, "mixed"), []
        for i, n in enumerate(news):
            paths.append(a_path(parents, int(layers[0].begin[i]), n, rng) if shape == "mixed" else sorted(rng.choice(n, int(rng.integers(0, n + 1)), replace=False).tolist()) if shape == "sparse" else
                         list(range(n // 2)) + [n - 1] * (n > 0))
        width = max(news)
        path = int32([p + [-1] * (width - len(p)) for p in paths])
        count = int32([len(p) for p in paths])
        want = [keep_reference(c, paths) for c in layers]
        handles = [c.wrap(ctx) for c in layers]
        ctx.clear_keep(handles, *layers[0].where, path, count)
        for c, (codes, scales), handle in zip(layers, want, handles):
            handle.check()
            for x, cd, sc in (("k", c.dev[0], c.dev[2]), ("v", c.dev[1], c.dev[3])):
                assert same_codes(cd.cpu(), codes[x]), (shape, x)
                assert torch.equal(sc.cpu().nan_to_num(nan=-1.0), scales[x].nan_to_num(nan=-1.0))
            handle.free()


def test_keep_in_many_layers_and_one(ctx):  # noqa: F811
    """More layers than a launch takes; a cache alone."""
    made = [Cache(ctx, [20], [9], 1, 64, 16, 50 + k) for k in range(35)]
    for c in made:
        c.table = made[0].table
        c.fill_new()
    want = [keep_reference(c, [[0, 3, 8]]) for c in made]
    handles = [c.wrap(ctx) for c in made]
    ctx.clear_keep(handles[:34], *made[0].where, int32([[0, 3, 8] + [-1] * 6]), int32([3]))
    ctx.clear_keep(handles[34], *made[0].where, int32([[0, 3, 8] + [-1] * 6]), int32([3]))
    for c, (codes, _), handle in zip(made, want, handles):
        assert same_codes(c.dev[0].cpu(), codes["k"]) and same_codes(c.dev[1].cpu(), codes["v"])
        handle.free()


def test_keep_of_some_of_a_batchs_sequences(ctx):  # noqa: F811
    """Rows of a batch's arrays: their tokens begin behind those of the rows before."""
    c = Cache(ctx, [20, 30, 9, 41], [64, 50, 5, 7], 2, 64, 16, 8)
    c.fill_new()
    paths = [[], [0, 7, 8, 49], [1, 4], []]
    codes, scales = keep_reference(c, paths)
    cache = c.wrap(ctx)
    table, begin, lengths = c.where
    path, count = int32([p + [-1] * (50 - len(p)) for p in paths[1:3]]), int32([4, 2])
    ctx.clear_keep(cache, table[1:3], begin[1:4], lengths[1:3], path, count)
    cache.check()
    for x, cd, sc in (("k", c.dev[0], c.dev[2]), ("v", c.dev[1], c.dev[3])):
        assert same_codes(cd.cpu(), codes[x]) and torch.equal(sc.cpu().nan_to_num(nan=-1.0), scales[x].nan_to_num(nan=-1.0))
    cache.free()


def test_paths_and_pages_that_do_not_fit_leave_the_sequence_out(ctx):  # noqa: F811
    from paper_2509_09424_amd import EnsiError
    c = Cache(ctx, [20, 30], [9, 9], 1, 64, 16, 7)
    c.fill_new()
    good = [0, 2, 5, 8] + [-1] * 5
    codes, scales = keep_reference(c, [good[:4], []])
    for bad, n in (([1, 1, 2], 3), ([2, 1, 5], 3), ([0, 3, 9], 3), ([-1, 3, 5], 3), ([0, 2, 5], 10), ([0, 2, 5], -1), ([0, 2, 2 ** 31 - 1], 3), ([0, -2 ** 31, 5], 3), ([0, 2, 5], 2 ** 31 - 1)):
        cache = c.wrap(ctx)
        ctx.clear_keep(cache, *c.where, int32([good, bad + [-1] * 6]), int32([4, n]))
        with pytest.raises(EnsiError, match="trees or paths"):
            cache.check()
        assert same_codes(c.dev[0].cpu(), codes["k"]) and torch.equal(c.dev[3].cpu().nan_to_num(nan=-1.0), scales["v"].nan_to_num(nan=-1.0))
        cache.free()
    cache = c.wrap(ctx)
    table = c.where[0].clone()
    table[1, 2] = 10 ** 6  # places 32 .. 47
    ctx.clear_keep(cache, table, *c.where[1:], int32([good, good]), int32([4, 4]))
    with pytest.raises(EnsiError, match="page numbers"):
        cache.check()
    assert same_codes(c.dev[0].cpu(), codes["k"])
    cache.free()
    # a sequence whose new tokens do not fit the path's width, noted in every cache
    made = [Cache(ctx, [20, 30], [9, 9], heads, 64, 16, 7) for heads in (1, 3, 1, 1, 2)]
    caches = [x.wrap(ctx) for x in made]
    ctx.clear_keep(caches, *c.where, int32([good[:8], good[:8]]), int32([4, 0]))
    for x, cache in zip(made, caches):
        with pytest.raises(EnsiError, match="do not fit the arguments"):
            cache.check()
        assert same_codes(x.dev[0].cpu(), x.codes["k"])
        cache.free()


def test_keep_rounds_every_code_as_torch_does(ctx):  # noqa: F811
    """All codes, moved beside a token whose scale is 1, 2, 8 or 2^20 times theirs, and NaN."""
    for power in (0, 1, 3, 20):
        c = Cache(ctx, [14], [18], 4, 64, 16, 3)
        c.fill_new()
        for x in "kv":
            one, two = int(c.table[0, 0]), int(c.table[0, 1])
            c.scales[x][one, :, 0], c.scales[x][two, :, 0] = 2.0 ** power, 1.0
            c.codes[x][two, :, 15] = torch.arange(256, dtype=torch.uint8).reshape(4, 64)
        want = keep_reference(c, [[0, 17]])
        cache = c.wrap(ctx)
        ctx.clear_keep(cache, *c.where, int32([[0, 17] + [-1] * 16]), int32([2]))
        cache.check()
        assert same_codes(c.dev[0].cpu(), want[0]["k"]) and same_codes(c.dev[1].cpu(), want[0]["v"])
        cache.free()


# ---- fork -------------------------------------------------------------------------------------------------------------------


def fork_reference(c, lengths, source, fresh):
    codes, scales = {x: t.clone() for x, t in c.codes.items()}, {x: t.clone() for x, t in c.scales.items()}
    table, width = [], c.table.shape[1]
    for s, f in zip(source, fresh):
        full, rest = divmod(lengths[s], c.page)
        table.append((c.table[s, :full].tolist() + [f] + [-1] * width)[:width])
        if rest:
            used, one = -(-rest // 16), int(c.table[s, full])
            for x in "kv":
                codes[x][f, :, :16 * used], scales[x][f, :, :used] = c.codes[x][one, :, :16 * used], c.scales[x][one, :, :used]
    return table, codes, scales


@pytest.mark.parametrize("ctxs, source, heads, dim, page", [([1], [0], 1, 64, 16), ([100, 0, 64, 37], [0, 0, 0, 3, 1, 2, 3], 2, 128, 64), ([5, 1000], [1, 1, 0], 3, 96, 16), ([250, 127, 129], [2, 1, 0, 0], 1, 256, 128),
                                                            ([48, 47, 49], [0, 1, 2] * 20, 4, 192, 48)])
def test_fork(ctx, ctxs, source, heads, dim, page):  # noqa: F811
    layers = []
    for k in range(2):
        c = Cache(ctx, ctxs, [0] * len(ctxs), heads + k, dim, page, 11 + k)
        used = c.codes["k"].shape[0]
        for x in "kv":  # pages for the rows
            c.codes[x] = torch.cat([c.codes[x], torch.full((len(source), heads + k, page, dim), 0x55, dtype=torch.uint8)])
            c.scales[x] = torch.cat([c.scales[x], torch.full((len(source), heads + k, page // 16), 7.0)])
        layers.append(c)
        c.table = layers[0].table
    fresh = (used + torch.randperm(len(source), generator=c.g)).tolist()
    # rows without a begun page may go without one; one goes on in the page it has
    for i, s in enumerate(source):
        if ctxs[s] % page == 0 and i % 2:
            fresh[i] = -1
    last = max(i for i, s in enumerate(source) if s == source[0])
    if ctxs[source[0]] % page:
        fresh[last] = int(c.table[source[0], ctxs[source[0]] // page])
    handles = [c.wrap(ctx) for c in layers]
    wide = torch.full((len(source), layers[0].table.shape[1] + 2), 77, dtype=torch.int32, device="cuda")
    out = wide[:, :-2]
    _, lengths = ctx.clear_fork(handles, layers[0].where[0], layers[0].where[2], int32(source), int32(fresh), table_out=out)
    for c, handle in zip(layers, handles):
        handle.check()
        table, codes, scales = fork_reference(c, ctxs, source, fresh)
        assert out.tolist() == table and lengths.tolist() == [ctxs[s] for s in source] and (wide[:, -2:] == 77).all()
        for x, cd, sc in (("k", c.dev[0], c.dev[2]), ("v", c.dev[1], c.dev[3])):
            assert torch.equal(cd.cpu(), codes[x]) and torch.equal(sc.cpu().nan_to_num(nan=-1.0), scales[x].nan_to_num(nan=-1.0))
        handle.free()


def test_forks_that_do_not_fit_leave_the_row_out(ctx):  # noqa: F811
    from paper_2509_09424_amd import EnsiError
    c = Cache(ctx, [20, 16, 40], [0, 0, 0], 1, 64, 16, 12)
    pages = c.codes["k"].shape[0]
    for x in "kv":
        c.codes[x] = torch.cat([c.codes[x], torch.full((4, 1, 16, 64), 0x55, dtype=torch.uint8)])
        c.scales[x] = torch.cat([c.scales[x], torch.full((4, 1, 1), 7.0)])
    width = c.table.shape[1]
    for source, fresh, bad in (([0, 0, 0], [pages, pages, pages + 1], [1]), ([0, 3, -1], [pages, pages + 1, pages + 2], [1, 2]), ([0, 2, 1], [-1, pages + 4, -1], [0, 1]), ([1, 0, 2], [pages, pages + 1, 2 ** 31 - 1], [2]),
                               ([1, 0, 1], [pages, pages, pages], [1, 2]), ([2 ** 31 - 1, -2 ** 31, 0], [pages, pages + 1, -2 ** 31], [0, 1, 2])):
        cache = c.wrap(ctx)
        table, lengths = ctx.clear_fork(cache, c.where[0], c.where[2], int32(source), int32(fresh))
        with pytest.raises(EnsiError, match="page numbers|do not fit"):
            cache.check()
        for i, (s, f) in enumerate(zip(source, fresh)):
            if i in bad:
                assert lengths[i] == 0 and table[i].tolist() == [-1] * width
            else:
                assert lengths[i] == c.ctxs[s] and table[i].tolist() == fork_reference(c, c.ctxs, [s], [f])[0][0]
        cache.free()
    # lengths that the table does not hold, and a page of the source outside the cache
    cache = c.wrap(ctx)
    table = c.where[0].clone()
    table[2, 2] = -5
    got, lengths = ctx.clear_fork(cache, table, int32([20, 16 * width + 1, 40]), int32([0, 1, 2]), int32([pages, pages + 1, pages + 2]))
    with pytest.raises(EnsiError, match="page numbers.*do not fit"):
        cache.check()
    assert lengths.tolist() == [20, 0, 0] and (got[1:] == -1).all()
    cache.free()


def test_fork_of_a_full_table(ctx):  # noqa: F811
    """No place is left behind the pages: fresh pages are not needed."""
    c = Cache(ctx, [32], [0], 1, 64, 16, 13)
    cache = c.wrap(ctx)
    table, lengths = ctx.clear_fork(cache, c.where[0][:, :2].contiguous(), c.where[2], int32([0, 0]), int32([-1, -1]))
    cache.check()
    assert table.tolist() == [c.table[0, :2].tolist()] * 2 and lengths.tolist() == [32, 32]
    assert not math.isnan(float(c.dev[2][int(c.table[0, 0])].sum()))
    cache.free()
