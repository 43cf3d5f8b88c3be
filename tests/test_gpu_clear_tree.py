"""Append and attention of trees of drafted tokens against their definitions in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_clear import TYPES, U32, Cache, append_reference, attention_near, ctx, half_step, same_codes, strided, turn32  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def trees(news, seed, shape="mixed"):
    """Parents of each sequence, one after the other."""
    rng, parents = np.random.default_rng(seed), []
    for n in news:
        t = np.arange(n)
        if shape == "chain":
            p = t - 1
        elif shape == "roots":
            p = np.full(n, -1)
        elif shape == "star":
            p = np.where(t > 0, 0, -1)
        else:
            p = np.array([-1 if i == 0 or rng.random() < 0.05 else max(0, i - 1 - int(rng.random() ** 2 * 6)) for i in t])
        parents.append(p)
    return torch.from_numpy(np.concatenate(parents).astype(np.int32))


def lines(parents, first, n):
    """Of each token of a sequence: its ancestors and itself, the nearest first."""
    out = []
    for t in range(n):
        line = [t]
        while int(parents[first + line[-1]]) >= 0:
            line.append(int(parents[first + line[-1]]))
        out.append(line)
    return out


def tree_reference(c, q, parents, cap, window, score, bias):
    group = q.shape[1] // c.heads
    out, size, top = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
    for i, (ctx_len, new) in enumerate(zip(c.ctxs, c.news)):
        first = int(c.begin[i])
        own = lines(parents, first, new)
        for h in range(c.heads):
            k, v = c.values("k", i, h), c.values("v", i, h)
            for t in range(new):
                reach = window or ctx_len + new
                seen = list(range(max(0, ctx_len + len(own[t]) - reach), ctx_len)) + [ctx_len + a for a in own[t][:reach]]
                for j in range(h * group, (h + 1) * group):
                    s = k[seen] @ q[first + t, j].double() / math.sqrt(c.dim)
                    top[first + t, j] = s.abs().max()
                    if cap:
                        s = cap * torch.tanh(s / cap)
                    p = torch.softmax(s, 0) if score == "softmax" else torch.sigmoid(s + bias)
                    out[first + t, j], size[first + t, j] = p @ v[seen], p @ v[seen].abs()
    return out, size, top


def tree_near(c, kind, got, q, parents, cap=0.0, window=0, score="softmax", bias=0.0):
    """The bounds of a chain's attention (attention_near)."""
    out, size, top = tree_reference(c, q, parents, cap, window, score, bias)
    n = max(a + b for a, b in zip(c.ctxs, c.news))
    weight = (2.0 ** -11 if kind == "bf16" else 2.0 ** -21) + n * U32 + (top[..., None] * 8 + 16 + (4 * cap if cap else 0)) * 2 * U32
    bound = half_step(kind) * out.abs() * (1 + 2.0 ** -7) + weight * size + n * 2.0 ** -25 * size.amax(2, keepdim=True) * 64 + torch.finfo(TYPES[kind]).smallest_normal * 2.0 ** -7
    off = (got.cpu().double() - out).abs()
    assert (off <= bound).all(), (off / bound).max()


CASES = [
    # ctxs, news, heads, group, dim, page, cap, window, score, shape
    ([0], [1], 1, 1, 64, 16, 0.0, 0, "softmax", "mixed"),
    ([31, 0, 500], [7, 1, 3], 2, 4, 128, 64, 0.0, 0, "softmax", "mixed"),
    ([1000, 77, 16, 15], [16, 16, 0, 16], 1, 8, 96, 16, 30.0, 100, "softmax", "mixed"),
    ([300], [64], 5, 3, 256, 128, 0.0, 17, "sigmoid", "mixed"),
    ([0, 20, 130], [50, 0, 7], 2, 1, 96, 16, 20.0, 33, "sigmoid", "mixed"),
    ([5], [64], 1, 5, 128, 48, 0.0, 0, "softmax", "chain"),
    ([64, 3], [40, 33], 2, 2, 64, 32, 5.0, 1, "softmax", "mixed"),
    ([100], [63], 1, 2, 192, 16, 0.0, 5, "softmax", "chain"),
    ([2500], [3], 1, 20, 128, 64, 0.0, 0, "softmax", "star"),
    ([33], [64], 1, 1, 256, 64, 0.0, 40, "softmax", "roots"),
    ([200, 0], [31, 60], 1, 4, 64, 16, 0.0, 0, "sigmoid", "star"),
    ([0, 1, 2], [64, 64, 64], 1, 2, 128, 16, 0.0, 3, "softmax", "mixed"),
    ([4000], [20], 2, 3, 128, 64, 0.0, 1500, "softmax", "mixed"),
    ([1500, 900], [12, 9], 4, 4, 192, 32, 7.0, 0, "sigmoid", "mixed"),
    ([31, 32, 33, 15], [33, 32, 31, 17], 2, 1, 64, 16, 0.0, 0, "softmax", "mixed"),
]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("ctxs, news, heads, group, dim, page, cap, window, score, shape", CASES)
def test_attention(ctx, kind, ctxs, news, heads, group, dim, page, cap, window, score, shape):  # noqa: F811
    c = Cache(ctx, ctxs, news, heads, dim, page, sum(ctxs) + sum(news) + dim)
    c.fill_new()
    parents = trees(news, sum(ctxs) + dim, shape)
    q = (torch.randn(c.tokens, heads * group, dim, generator=c.g) / 16).to(TYPES[kind])
    cache = c.wrap(ctx)
    out = strided(torch.full_like(q, 9.0), 5)
    bias = -math.log(max(ctxs) + max(news)) if score == "sigmoid" else 0.0
    ctx.clear_attention(cache, *c.where, strided(q, 3), out, cap=cap, window=window, score=score, bias=bias, max_new=max(news), max_length=max(a + b for a, b in zip(ctxs, news)), parents=parents.cuda())
    cache.check()
    tree_near(c, kind, out, q, parents, cap, window, score, bias)
    if shape == "chain":
        attention_near(c, kind, out, q, cap, window, score, bias)
    # the bounds that a caller gives do not change what is computed, only how it is split
    again = ctx.clear_attention(cache, *c.where, strided(q, 3), None, cap=cap, window=window, score=score, bias=bias, parents=parents.cuda())
    tree_near(c, kind, again, q, parents, cap, window, score, bias)
    cache.free()


def test_unseen_places_have_no_part(ctx):  # noqa: F811
    """NaN in keys and values of tokens that are no ancestors, behind the last one, before the window, and on pages that were given back; a token that sees one is NaN there."""
    c = Cache(ctx, [100], [12], 1, 64, 16, 5)
    c.fill_new()
    parents = torch.tensor([-1, 0, 0, 1, 2, 3, 4, 5, 6, 7, 8, 2], dtype=torch.int32)
    q = (torch.randn(12, 2, 64, generator=c.g) / 16).bfloat16()
    own = lines(parents, 0, 12)
    place = lambda p: (int(c.table[0, p // 16]), 0, p % 16)  # noqa: E731
    for x in "kv":
        c.codes[x][place(102)] = 0x7f  # token 2: only its line sees it
    c.codes["v"][place(60)][7] = 0x7f  # a cached value before every window of 30
    window = 30
    table = c.table.clone()
    table[0, :4] = 10 ** 6  # places before 64: given back
    cache = c.wrap(ctx)
    got = ctx.clear_attention(cache, table.cuda(), *c.where[1:], q.cuda(), window=window, parents=parents.cuda()).cpu()
    cache.check()
    sees = [2 in line for line in own]
    assert got[sees].isnan().all() and got[[not s for s in sees]].isfinite().all()
    c.codes["k"][place(102)] = 0
    c.codes["v"][place(102)] = 0
    c.codes["v"][place(102)][3] = 0xff  # one value
    c.codes["v"][place(60)][7] = 0
    cache.free()
    cache = c.wrap(ctx)
    got = ctx.clear_attention(cache, *c.where, q.cuda(), window=window, parents=parents.cuda()).cpu()
    assert got[sees][..., 3].isnan().all() and torch.cat([got[sees][..., :3], got[sees][..., 4:]], -1).isfinite().all() and got[[not s for s in sees]].isfinite().all()
    keep = [t for t in range(12) if not sees[t]]
    out, size, _ = tree_reference(c, q, parents, 0.0, window, "softmax", 0.0)
    assert ((got.double() - out).abs()[keep] <= (2.0 ** -8 + 2.0 ** -10) * size.abs()[keep]).all()
    cache.free()


def test_trees_and_pages_that_do_not_fit_are_left_out(ctx):  # noqa: F811
    from paper_2509_09424_amd import EnsiError
    c = Cache(ctx, [40, 20, 33], [5, 6, 4], 2, 64, 16, 6)
    c.fill_new()
    q = (torch.randn(c.tokens, 2, 64, generator=c.g) / 16).bfloat16()
    good = trees(c.news, 1)
    for at, bad in ((7, 2), (7, 5), (7, -2), (5, 0), (10, 2 ** 31 - 1), (6, -2 ** 31)):
        parents = good.clone()
        parents[at] = bad
        cache = c.wrap(ctx)
        out = torch.full_like(q, 9.0).cuda()
        ctx.clear_attention(cache, *c.where, q.cuda(), out, parents=parents.cuda())
        with pytest.raises(EnsiError, match="trees or paths"):
            cache.check()
        whole = ctx.clear_attention(cache, *c.where, q.cuda(), parents=good.cuda()).cpu()
        out = out.cpu()
        assert (out[5:11] == 9).all() and torch.equal(out[:5], whole[:5]) and torch.equal(out[11:], whole[11:])
        before = [t.clone() for t in c.dev]
        k = torch.randn(c.tokens, 2, 64, device="cuda").bfloat16()
        ctx.clear_append(cache, *c.where, k, k, None, None, parents=parents.cuda())
        with pytest.raises(EnsiError, match="trees or paths"):
            cache.check()
        for i in range(20, 26):
            one, r = int(c.table[1, i // 16]), i % 16
            assert torch.equal(c.dev[0][one, :, r], before[0][one, :, r])
        cache.free()
    # all pages outside the cache: rows of 0; of one sequence's last page: its earlier keys remain
    cache = c.wrap(ctx)
    table = c.where[0].clone()
    table[1] = -1
    table[0, 2] = 10 ** 6
    got = ctx.clear_attention(cache, table, *c.where[1:], q.cuda(), parents=good.cuda()).cpu()
    with pytest.raises(EnsiError, match="page numbers"):
        cache.check()
    assert (got[5:11] == 0).all() and got[:5].isfinite().all() and (got[:5] != 0).any()
    # a rotation that the positions do not hold
    cos = torch.ones(42, 32, device="cuda")
    k = torch.randn(c.tokens, 2, 64, device="cuda").bfloat16()
    chain = trees(c.news, 0, "chain").cuda()
    ctx.clear_append(cache, *c.where, k, k, cos, cos, parents=trees(c.news, 0, "star").cuda())
    cache.check()  # places to 44, positions to 41
    ctx.clear_append(cache, *c.where, k, k, cos, cos, parents=chain)
    with pytest.raises(EnsiError, match="do not fit the arguments"):
        cache.check()
    cache.free()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("ctxs, news, q_heads, heads, dim, rot, pairs, page, shape", [
    ([0], [1], 1, 1, 64, 64, "half", 16, "mixed"), ([15, 16, 17, 0, 100], [9, 1, 64, 20, 33], 4, 2, 128, 128, "half", 64, "mixed"), ([0, 3, 40], [33, 0, 17], 3, 3, 96, 48, "neighbours", 16, "star"),
    ([7], [64], 8, 1, 256, 256, "neighbours", 32, "mixed"), ([1, 250], [31, 14], 2, 2, 192, 96, "half", 128, "chain"), ([12], [20], 2, 1, 128, 0, "half", 16, "mixed")])
def test_append(ctx, kind, ctxs, news, q_heads, heads, dim, rot, pairs, page, shape):  # noqa: F811
    """Rotated by the length and the depth, stored one behind the other."""
    c = Cache(ctx, ctxs, news, heads, dim, page, sum(ctxs) + dim)
    parents = trees(news, dim, shape)
    q = torch.randn(c.tokens, q_heads, dim, generator=c.g).to(TYPES[kind])
    both = (torch.randn(c.tokens, 2 * heads, dim, generator=c.g) * 2.0 ** torch.randint(-6, 7, (c.tokens, 2 * heads, 1), generator=c.g).float()).to(TYPES[kind])
    place = np.concatenate([[a + len(line) - 1 for line in lines(parents, int(c.begin[i]), n)] for i, (a, n) in enumerate(zip(ctxs, news))]).astype(int)
    positions = int(place.max()) + 1
    angle = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(0, max(rot, 2), 2) / max(rot, 2))
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    turned = turn32(both[:, :heads], cos[place][:, None], sin[place][:, None], rot, pairs) if rot else both[:, :heads].float().numpy()
    codes, scales = append_reference(c, torch.from_numpy(turned), both[:, heads:], None, None, 0, pairs)
    cache, dev = c.wrap(ctx), both.cuda()
    turn = (torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()) if rot else (None, None)
    got = ctx.clear_append(cache, *c.where, dev[:, :heads], dev[:, heads:], *turn, q=strided(q, 3), pairs=pairs, parents=parents.cuda())
    cache.check()
    for x, (cd, sc) in zip("kv", ((c.dev[0], c.dev[2]), (c.dev[1], c.dev[3]))):
        assert same_codes(cd.cpu(), codes[x]) and torch.equal(sc.cpu().nan_to_num(nan=-1.0), scales[x].nan_to_num(nan=-1.0))
    want = torch.from_numpy(turn32(q, cos[place][:, None], sin[place][:, None], rot, pairs)).to(TYPES[kind]) if rot else q
    assert torch.equal(got.cpu(), want)
    cache.free()


def test_many_sequences_and_a_long_one(ctx):  # noqa: F811
    """More parts than rows, and more sequences than workgroups find room for, on the GPU in 64 bits a head at a time."""
    for ctxs, news, heads, group, dim in (([30000], [13], 2, 4, 128), (list(range(0, 1200, 7)), [1 + i % 9 for i in range(172)], 2, 2, 64)):
        c = Cache(ctx, [0], [1], heads, dim, 64, 1)
        c.ctxs, c.news = ctxs, news
        need = [-(-(a + n) // 64) for a, n in zip(ctxs, news)]
        pages = sum(need)
        c.table = torch.zeros(len(ctxs), max(need), dtype=torch.int32)
        order, at = torch.randperm(pages, generator=c.g).int(), 0
        for i, k in enumerate(need):
            c.table[i, :k] = order[at:at + k]
            at += k
        for x in "kv":
            c.codes[x] = (torch.randn(pages, heads, 64, dim, generator=c.g) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            c.scales[x] = 2.0 ** torch.randint(-8, -5, (pages, heads, 4), generator=c.g).float()
        c.begin = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32)
        c.lengths, c.tokens = torch.tensor(ctxs, dtype=torch.int32), sum(news)
        parents = trees(news, 3)
        q = torch.randn(c.tokens, heads * group, dim, generator=c.g).bfloat16()
        cache = c.wrap(ctx)
        got = ctx.clear_attention(cache, *c.where, q.cuda(), max_new=max(news), max_length=max(a + b for a, b in zip(ctxs, news)), parents=parents.cuda())
        cache.check()
        tree_near(c, "bf16", got, q, parents)
        assert torch.equal(got, ctx.clear_attention(cache, *c.where, q.cuda(), max_new=max(news), max_length=max(a + b for a, b in zip(ctxs, news)), parents=parents.cuda()))
        cache.free()


def test_batches_without_new_tokens(ctx):  # noqa: F811
    """No sequences, and sequences with nothing new: an empty tensor of parents is one."""
    c = Cache(ctx, [20, 3], [0, 0], 2, 64, 16, 4)
    cache = c.wrap(ctx)
    before = [t.clone() for t in c.dev]
    x = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    parents = torch.empty(0, dtype=torch.int32, device="cuda")
    for n in (2, 0):
        table, begin, lengths = c.where[0][:n], c.where[1][:n + 1], c.where[2][:n]
        ctx.clear_append(cache, table, begin, lengths, x, x, None, None, parents=parents)
        assert ctx.clear_attention(cache, table, begin, lengths, x, parents=parents).shape == (0, 2, 64)
        path, count, following = ctx.clear_accept(begin, parents, parents, parents, max_new=0)
        assert path.shape == (n, 0) and count.tolist() == [0] * n and following.tolist() == [-1] * n
        ctx.clear_keep(cache, table, begin, lengths, path, count)
    cache.check()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, c.dev))
    cache.free()


@pytest.mark.parametrize("new, group, dim, score", [(5, 3, 64, "softmax"), (20, 4, 64, "sigmoid"), (3, 8, 192, "softmax")])
def test_a_long_sequence_in_many_parts(ctx, new, group, dim, score):  # noqa: F811
    """61440 cached tokens, 60 times the same 64 pages, in up to 64 parts of a row's keys."""
    c = Cache(ctx, [1024], [new], 1, dim, 16, dim + new)
    c.fill_new()
    c.table = torch.cat([c.table[:, :64].repeat(1, 60), c.table[:, 64:]], 1)
    c.ctxs, c.lengths = [61440], torch.tensor([61440], dtype=torch.int32)
    parents = trees([new], 3)
    q = (torch.randn(new, group, dim, generator=c.g) / 16).bfloat16()
    cache = c.wrap(ctx)
    bias = -math.log(61440) if score == "sigmoid" else 0.0
    out = ctx.clear_attention(cache, *c.where, q.cuda(), score=score, bias=bias, max_length=61440 + new, parents=parents.cuda())
    cache.check()
    tree_near(c, "bf16", out, q, parents, score=score, bias=bias)
    cache.free()
