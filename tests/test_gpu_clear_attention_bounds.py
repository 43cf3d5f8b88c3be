"""Attention on clear activations against 64 bits with bounds for each place of each row: of the row's own keys and of that place's own terms, so that what a row's
largest contribution would hide is seen where that contribution has no part."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_clear import CASES, TYPES, U32, Cache, ctx, e4m3, half_step  # noqa: E402, F401

PAIR = 2.0 ** -16  # weights in two terms of bf16: half a step of one of them, of half a step of the other


def definition(c, q, i, h, j, cap, window, score, bias):
    """Of sequence i and query head j over key head h, in 64 bits: outputs, the sum of their terms' sizes, and what the weights may be off by beside the roundings to 16 bits, relatively."""
    first, new = int(c.begin[i]), c.news[i]
    n = c.ctxs[i] + new
    k, v, x = c.values("k", i, h).cuda(), c.values("v", i, h).cuda(), q[first:first + new, j].cuda().double()
    root = 1 / math.sqrt(c.dim)
    t, sizes = x @ k.T * root, x.abs() @ k.abs().T * root
    at, key = torch.arange(n - new, n, device="cuda")[:, None], torch.arange(n, device="cuda")
    dark = key > at
    if window:
        dark = dark | (key <= at - window)
    t, sizes = t.masked_fill(dark, 0), sizes.masked_fill(dark, 0)
    raw = t.abs().amax(1, keepdim=True)
    if cap:
        t = cap * torch.tanh(t / cap)
    p = torch.softmax(t.masked_fill(dark, -math.inf), 1) if score == "softmax" else torch.sigmoid(t + bias).masked_fill(dark, 0)
    v = v.masked_fill(~(p > 0).any(0)[:, None], 0)  # (NaN where nobody looks)
    seen = (~dark).sum(1, keepdim=True)
    # a score: `dim` products added in 32 bits, each addition a whole step of the sum of sizes at most; five roundings of its own (factor, scale, cap); the exponent's argument has four more at the
    # size of scores, references and lifts in units of log2 e
    if cap:  # the exponential, 1 + it, its reciprocal and the difference from 1, of half a cap at least: 5.5 of U32 of the cap; or seven terms of a series
        off = 12 * U32 * raw
    else:
        off = 0
    scale = c.scales["v"].nan_to_num(1.0, 1.0, 1.0).clamp(2.0 ** -64, 2.0 ** 120).log2().abs().max()
    off = off + 2 * U32 * (c.dim * sizes.amax(1, keepdim=True) + 5 * raw) + 4 * U32 * (1.5 * (t.abs().amax(1, keepdim=True) + abs(bias)) + float(scale) + 70)
    # the running reference moves once a tile of 32 keys at most, six roundings each time; then sums over the row's keys, of weights and of products; functions to two steps
    return p @ v, p @ v.abs(), 2 * off + U32 * (6 * seen / 32 + 2 * seen + 32)


def check(c, kind, got, q, cap=0.0, window=0, score="softmax", bias=0.0, heads=None):
    worst = 0.0
    for i in range(len(c.ctxs)):
        first, new = int(c.begin[i]), c.news[i]
        group = q.shape[1] // c.heads
        for j in () if not new else range(q.shape[1]) if heads is None else heads:
            out, size, off = definition(c, q, i, j // group, j, cap, window, score, bias)
            bound = half_step(kind) * (1 + 2.0 ** -7) * out.abs() + (PAIR + off) * size + torch.finfo(TYPES[kind]).smallest_normal * half_step(kind)
            ratio = ((got[first:first + new, j].cuda().double() - out).abs() / bound).max().item()
            assert ratio <= 1, (i, j, ratio)  # (also where it is NaN)
            worst = max(worst, ratio)
    return worst


def longest(c):
    return {"max_new": max(c.news), "max_length": max(a + b for a, b in zip(c.ctxs, c.news))}


PROMPTS = [([70, 0], [1800, 1000], 8, 4, 64, 16, 0.0, 0, "softmax"), ([200], [1500], 8, 4, 128, 64, 0.0, 0, "softmax"), ([33], [1501], 8, 2, 96, 32, 20.0, 300, "softmax"),
           ([10], [1500], 4, 6, 192, 16, 0.0, 0, "sigmoid"), ([100], [1450], 8, 4, 256, 64, 0.0, 500, "softmax"), ([5, 300, 40], [1500, 0, 911], 8, 2, 64, 48, 9.0, 0, "sigmoid")]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("ctxs, news, heads, group, dim, page, cap, window, score", CASES + PROMPTS)
def test_every_place(ctx, kind, ctxs, news, heads, group, dim, page, cap, window, score):
    c = Cache(ctx, ctxs, news, heads, dim, page, sum(ctxs) + 3 * sum(news) + dim)
    c.fill_new()
    q = (torch.randn(c.tokens, heads * group, dim, generator=c.g) / 16).to(TYPES[kind])
    cache = c.wrap(ctx)
    bias = -math.log(max(ctxs) + max(news)) if score == "sigmoid" else 0.0
    got = ctx.clear_attention(cache, *c.where, q.cuda(), cap=cap, window=window, score=score, bias=bias, **longest(c))
    cache.check()
    check(c, kind, got, q, cap, window, score, bias, None if group * heads < 8 else range(0, heads * group, 3))
    cache.free()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("news", [[30], [1500, 1200, 700]])
def test_values_that_cancel(ctx, kind, news):
    """Neighbouring tokens have opposite values: the outputs are differences of nearly equal weights, whose roundings show.  Early tokens see few keys."""
    c = Cache(ctx, [0] * len(news), news, 8 if len(news) > 1 else 2, 64, 16, 31)
    c.fill_new(powers=(-3, -2))
    for i, n in enumerate(news):
        for p in range(1, n, 2):
            one, r = int(c.table[i, p // 16]), p % 16
            c.codes["v"][one, :, r] = c.codes["v"][one, :, r - 1] ^ 0x80
    q = (torch.randn(c.tokens, 4 * c.heads, 64, generator=c.g) / 1024).to(TYPES[kind])
    cache = c.wrap(ctx)
    got = ctx.clear_attention(cache, *c.where, q.cuda(), **longest(c))
    check(c, kind, got, q, heads=range(0, 4 * c.heads, 3))
    cache.free()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("nats", [14, 18, 26, 40])
@pytest.mark.parametrize("ctxs, news, heads", [([700], [1], 1), ([3000], [1], 2), ([300], [40], 1), ([0], [1800], 16)])
def test_a_key_that_takes_all_and_gives_nothing(ctx, kind, nats, ctxs, news, heads):
    """The first token has e^nats times the weight of any other and values of 0 in half of the places: there the others are the result."""
    c = Cache(ctx, ctxs, news, heads, 64, 16, 100 + nats, powers=(0, 1))
    c.fill_new(powers=(0, 1))
    for i in range(len(c.table)):  # score = first element of the key (queries are 8 e_0): small, and `nats` for the first token
        for p in range(c.ctxs[i] + c.news[i]):
            c.codes["k"][int(c.table[i, p // 16]), :, p % 16, 0] = (torch.randn(heads, generator=c.g) * 0.3).to(torch.float8_e4m3fn).view(torch.uint8)
        one = int(c.table[i, 0])
        c.codes["k"][one, :, 0, 0] = torch.tensor([float(nats)]).to(torch.float8_e4m3fn).view(torch.uint8)
        c.codes["v"][one, :, 0, :32] = 0
        for b in range(1, -(-(c.ctxs[i] + c.news[i]) // 16)):
            c.scales["v"][int(c.table[i, b]), :, 0] = 2.0 ** 8
    q = torch.zeros(c.tokens, 4 * heads, 64)
    q[:, :, 0] = 8
    q = q.to(TYPES[kind])
    cache = c.wrap(ctx)
    got = ctx.clear_attention(cache, *c.where, q.cuda(), **longest(c))
    check(c, kind, got, q, heads=range(0, 4 * heads, 5))
    cache.free()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("news, heads", [([1], 1), ([90], 2), ([1700], 16)])
def test_scales_far_apart_and_zeros_beside_the_large_ones(ctx, kind, news, heads):
    """Value scales from 2^-60 to 2^100 (f16: 2^-4 to 2^6) in one sequence; the block with the largest has values in every other place only."""
    low, mid, high = (-60, -30, 100) if kind == "bf16" else (-9, -4, 6)
    c = Cache(ctx, [200], news, heads, 64, 16, 33)
    c.fill_new()
    for b in range((200 + news[0]) // 16 + 1):
        c.scales["v"][int(c.table[0, b]), :, 0] = 2.0 ** (low if b % 2 else mid)
    one = int(c.table[0, 2])
    c.scales["v"][one, :, 0] = 2.0 ** high
    c.codes["v"][one, :, :, ::2] = 0
    q = (torch.randn(c.tokens, 4 * heads, 64, generator=c.g) / 16).to(TYPES[kind])
    cache = c.wrap(ctx)
    got = ctx.clear_attention(cache, *c.where, q.cuda(), **longest(c))
    check(c, kind, got, q, heads=range(0, 4 * heads, 5))
    cache.free()


@pytest.mark.parametrize("exponent", [120, -64])
@pytest.mark.parametrize("news, heads", [([1], 1), ([40], 1), ([1700], 16)])
def test_scales_at_either_end(ctx, exponent, news, heads):
    """All value scales 2^120, or all 2^-64: the softmax's sum holds terms of e^-20 beside those of the largest score, which belong to a token without values."""
    c = Cache(ctx, [400], news, heads, 64, 16, 35, powers=(0, 1))
    c.fill_new(powers=(0, 1))
    for p in range(400 + news[0]):
        one, r = int(c.table[0, p // 16]), p % 16
        c.codes["k"][one, :, r, 0] = torch.tensor([20.0 if p == 5 else 0.25 * (p % 3)]).to(torch.float8_e4m3fn).view(torch.uint8)
        c.codes["v"][one, :, r] = 0 if p == 5 else torch.tensor([0.5 + p % 2]).to(torch.float8_e4m3fn).view(torch.uint8)
        c.scales["v"][one, :, r // 16] = 2.0 ** exponent
    q = torch.zeros(c.tokens, 4 * heads, 64)
    q[:, :, 0] = 8
    q = q.to(torch.bfloat16)
    cache = c.wrap(ctx)
    got = ctx.clear_attention(cache, *c.where, q.cuda(), **longest(c))
    check(c, "bf16", got, q, heads=range(0, 4 * heads, 5))
    cache.free()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("cap", [1e-40, 1e-3, 1.0, 30.0, 1e4, 1e6, 1e8, 3e38])
@pytest.mark.parametrize("ctxs, news, heads", [([900, 31], [1, 1], 1), ([0], [1700], 16)])
def test_caps_of_every_size(ctx, kind, score, cap, ctxs, news, heads):
    """Scores of deviation 2 under caps far below, near and far above them, where the cap leaves them as they are."""
    c = Cache(ctx, ctxs, news, heads, 64, 16, 41, powers=(0, 1))
    c.fill_new(powers=(0, 1))
    q = (torch.randn(c.tokens, 4 * heads, 64, generator=c.g) / 30).to(TYPES[kind])  # values of deviation 60, divided by 8
    cache = c.wrap(ctx)
    bias = -6.0 if score == "sigmoid" else 0.0
    got = ctx.clear_attention(cache, *c.where, q.cuda(), cap=cap, score=score, bias=bias, **longest(c))
    check(c, kind, got, q, cap, 0, score, bias, heads=range(0, 4 * heads, 7))
    cache.free()


@pytest.mark.parametrize("score, cap", [("softmax", 0.0), ("softmax", 9.0), ("sigmoid", 0.0)])
@pytest.mark.parametrize("ctxs, news, heads, window", [([300], [1], 1, 50), ([301, 64], [1, 1], 2, 17), ([290], [40], 1, 33), ([300], [1500], 16, 77), ([40], [1600], 16, 16), ([1000], [1], 1, 1)])
def test_pages_before_a_window_that_were_given_back(ctx, score, cap, ctxs, news, heads, window):
    """Pages that no row of a tile sees: whatever their place in the table and their scales hold, the results are the same, and nothing is reported."""
    c = Cache(ctx, ctxs, news, heads, 64, 16, 43 + window)
    c.fill_new()
    q = (torch.randn(c.tokens, 4 * heads, 64, generator=c.g) / 16).to(torch.bfloat16)
    bias = -4.0 if score == "sigmoid" else 0.0
    call = lambda cache, table: ctx.clear_attention(cache, table, *c.where[1:], q.cuda(), cap=cap, window=window, score=score, bias=bias, **longest(c))  # noqa: E731
    cache = c.wrap(ctx)
    clean = call(cache, c.where[0])
    cache.check()
    check(c, "bf16", clean, q, cap, window, score, bias, heads=range(0, 4 * heads, 7))
    given_back = [(i, b) for i, n in enumerate(c.ctxs) for b in range(max(0, (n - window + 1) // 16))]
    assert given_back
    spare = next(p for p in range(len(c.codes["k"])) if not (c.table == p).any())
    for what in (-1, 1 << 30, spare):
        for k_scale, v_scale in ((0.0, 0.0), (math.nan, math.nan), (math.inf, math.inf), (1.0, math.inf), (math.inf, 1.0)) if what == spare else ((1.0, 1.0),):
            table = c.table.clone()
            for i, b in given_back:
                table[i, b] = what
            cache.free()
            cache = c.wrap(ctx)
            c.dev[2][spare], c.dev[3][spare] = k_scale, v_scale
            got = call(cache, table.cuda())
            cache.check()
            assert torch.equal(got, clean), (what, k_scale, v_scale)
    cache.free()


@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("ctxs, news, heads", [([0], [1], 1), ([40], [1], 1), ([3000], [1], 1), ([30], [50], 2), ([0], [1700], 16)])
def test_scores_of_minus_infinity(ctx, cap, ctxs, news, heads):
    """Scores that overflow: rows with none but -inf have no softmax and are NaN (a cap turns -inf into minus itself, which is a score like any other), -inf beside finite
    scores is a weight of 0; a row whose pages are all outside the cache stays 0."""
    c = Cache(ctx, ctxs, news, heads, 64, 16, 51, powers=(0, 1))
    c.fill_new(powers=(0, 1))
    big = torch.tensor([256.0]).to(torch.float8_e4m3fn).view(torch.uint8)
    n = ctxs[0] + news[0]
    for p in range(n):
        c.codes["k"][int(c.table[0, p // 16]), :, p % 16] = 0
        c.codes["k"][int(c.table[0, p // 16]), :, p % 16, 0] = big
    group = 4
    q = torch.zeros(c.tokens, group * heads, 64)
    q[:, 1::group] = torch.randn(c.tokens, heads, 64, generator=c.g) / 16
    q[:, 0::group, 0], q[:, 2::group, 0] = -3e38, 3e38
    q = q.to(torch.bfloat16)
    cache = c.wrap(ctx)
    got = ctx.clear_attention(cache, *c.where, q.cuda(), cap=cap, **longest(c)).cpu()
    cache.check()
    assert got[:, 1::group].isfinite().all() and got[:, 3::group].isfinite().all()
    if cap:
        assert got.isfinite().all()
        check(c, "bf16", got, torch.where(q.abs() > 1e38, 0.0, q), cap)  # equal scores in either
        cache.free()
        return
    assert got[:, 0::group].isnan().all() and got[:, 2::group].isnan().all()
    if n > 1:  # the first token's key is 0: its score is 0 for every row, all others are -inf
        c.codes["k"][int(c.table[0, 0]), :, 0, 0] = 0
        cache.free()
        cache = c.wrap(ctx)
        got = ctx.clear_attention(cache, *c.where, q.cuda(), **longest(c)).cpu()
        first = e4m3(c.codes["v"][int(c.table[0, 0]), :, 0]) * c.scales["v"][int(c.table[0, 0]), :, 0, None]
        assert torch.equal(got[:, 0::group].float(), first.to(torch.bfloat16).float().expand(c.tokens, heads, 64))
    table = torch.full_like(c.table, -1)
    got = ctx.clear_attention(cache, table.cuda(), *c.where[1:], q.cuda(), **longest(c)).cpu()
    assert (got == 0).all()
    with pytest.raises(Exception, match="left out"):
        cache.check()
    cache.free()


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("news, heads", [([1], 1), ([1600], 16)])
def test_scores_near_the_largest_cap(ctx, sign, news, heads):
    """Scores of 2e38 under a cap of 3e38: all of a row's are equal, so the softmax is a mean."""
    c = Cache(ctx, [0], news, heads, 64, 16, 53, powers=(0, 1))
    c.fill_new(powers=(0, 1))
    for p in range(news[0]):
        c.codes["k"][int(c.table[0, p // 16]), :, p % 16] = torch.tensor([8.0] + [0.0] * 63).to(torch.float8_e4m3fn).view(torch.uint8)
    q = torch.zeros(c.tokens, 4 * heads, 64)
    q[:, :, 0] = sign * 2e38
    q = q.to(torch.bfloat16)
    cache = c.wrap(ctx)
    got = ctx.clear_attention(cache, *c.where, q.cuda(), cap=3e38, **longest(c))
    check(c, "bf16", got, torch.zeros_like(q), heads=range(0, 4 * heads, 5))  # equal scores
    cache.free()
