"""The decoder layer on clear activations against its definitions in 64 bits: norm with codes, ternary product, append to the paged 8-bit cache,
attention over it."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U32 = 2.0 ** -24  # half a step of 32 bits


def half_step(kind):
    return torch.finfo(TYPES[kind]).eps / 2


@pytest.fixture(scope="module")
def ctx():
    from paper_2509_09424_amd import Context
    c = Context(12, 36, 3, 37, 1, 1, 30)
    yield c
    c.close()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def strided(t, pad):
    """The same rows with `pad` more elements between them, on the GPU."""
    wide = torch.full((t.shape[0], math.prod(t.shape[1:]) + pad), 7.0 if t.is_floating_point() else 7).to(t.dtype)
    wide[:, :wide.shape[1] - pad] = t.reshape(t.shape[0], -1)
    return wide.cuda()[:, :wide.shape[1] - pad].unflatten(1, t.shape[1:]) if t.dim() > 2 else wide.cuda()[:, :wide.shape[1] - pad]


# ---- norm -------------------------------------------------------------------------------------------------------------------


def norm_reference(x, gain, residual, eps):
    """Codes from products of 32 bits, as the definition has them; the rest in 64."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    p = (h.float() * gain.float()).numpy()
    most = np.abs(p).max(1, keepdims=True)
    with np.errstate(all="ignore"):
        factor = np.float32(127) * (np.float32(1) / most)
        codes = np.where(most > 0, np.rint(p * factor), 0)
    h64 = h.double()
    root = 1 / torch.sqrt((h64 ** 2).mean(1) + eps)
    p64 = h64 * gain.double()
    return h, codes, p64.abs().amax(1) / 127 * root, p64 * root[:, None]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows, d, pad, residual", [(1, 1, 0, False), (1, 64, 0, True), (3, 7, 1, True), (5, 1000, 3, False), (2, 2561, 0, True), (1030, 129, 1, True), (1024, 2560, 0, True),
                                                    (1025, 4090, 8, False), (9, 8191, 1, True), (2, 20000, 0, True), (1, 32768, 0, False)])
def test_norm(ctx, kind, rows, d, pad, residual):
    g = gen(rows * d)
    x, r = torch.randn(rows, d, generator=g).to(TYPES[kind]), (torch.randn(rows, d, generator=g) * 3).to(TYPES[kind]) if residual else None
    gain = (1 + 0.2 * torch.randn(d, generator=g)).to(TYPES[kind])
    h, codes, scales, full = norm_reference(x, gain, r, 1e-5)
    sum_out = strided(torch.zeros_like(x), pad + 2) if residual else None
    out = strided(torch.zeros_like(x), pad)
    got, got_scales = ctx.clear_norm(strided(x, pad), gain.cuda(), residual=None if r is None else strided(r, pad + 1), eps=1e-5, sum_out=sum_out, out=out,
                                     codes=torch.full((rows, d), 55, dtype=torch.int8, device="cuda"))
    assert np.array_equal(got.cpu().numpy(), codes)
    # a sum of squares in 32 bits: a thread adds up to 64 of them in turn, then 10 levels; half of that through the root, and a few roundings more
    near = 64 * U32
    assert ((got_scales.cpu().double() - scales).abs() <= near * scales).all()
    assert ((out.cpu().double() - full).abs() <= (near + half_step(kind)) * full.abs() + torch.finfo(TYPES[kind]).tiny).all()
    if residual:
        assert torch.equal(sum_out.cpu(), h)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows, d, pad, residual", [(2050, 500, 1, True), (2049, 1023, 0, False), (2051, 2000, 3, True), (2049, 4089, 0, True), (1025, 1030, 5, True)])
def test_norm_of_many_rows(ctx, kind, rows, d, pad, residual):
    """A wave to a row, of every number of chunks."""
    test_norm(ctx, kind, rows, d, pad, residual)


@pytest.mark.parametrize("rows", [3, 1500])
def test_norm_in_place(ctx, rows):
    g = gen(rows)
    x, r, gain = torch.randn(rows, 300, generator=g), torch.randn(rows, 300, generator=g), torch.randn(300, generator=g)
    h, codes, _, full = norm_reference(x, gain, r, 1e-5)
    for into in ("x", "residual"):
        xd, rd = x.cuda(), r.cuda()
        got, _ = ctx.clear_norm(xd, gain.cuda(), residual=rd, sum_out={"x": xd, "residual": rd}[into], codes=torch.empty(rows, 300, dtype=torch.int8, device="cuda"))
        assert torch.equal({"x": xd, "residual": rd}[into].cpu(), h) and np.array_equal(got.cpu().numpy(), codes)
    xd = x.cuda()
    ctx.clear_norm(xd, gain.cuda(), out=xd)
    _, _, _, full = norm_reference(x, gain, None, 1e-5)
    assert torch.allclose(xd.cpu().double(), full, rtol=64 * U32 + U32, atol=1e-30)


def test_norm_of_extreme_rows(ctx):
    """Rows of zeros, of the smallest numbers, with an infinity or NaN, and with squares that leave the range; their neighbours are untouched."""
    x = torch.ones(8, 40)
    x[0] = 0
    x[1, 3], x[2, 5] = math.inf, math.nan
    x[3] = 1e-38 * torch.arange(40)
    x[4] = 3e19
    x[5] = 1e-44
    x[6] = -0.0
    x[7] = 2.0 ** torch.arange(40)
    gain = torch.ones(40)
    out = torch.empty(8, 40, device="cuda")
    codes, scales = ctx.clear_norm(x.cuda(), gain.cuda(), out=out, eps=1e-5, codes=torch.empty(8, 40, dtype=torch.int8, device="cuda"))
    codes, scales, out = codes.cpu().numpy(), scales.cpu().numpy(), out.cpu().numpy()
    for bad in (1, 2, 4):
        assert np.isnan(scales[bad]) and np.isnan(out[bad]).all() and not codes[bad].any()
    for zero in (0, 6):
        assert scales[zero] == 0 and not codes[zero].any() and not out[zero].any()
    assert np.array_equal(codes[3], np.rint(np.arange(40) * 127 / 39)) and np.array_equal(codes[5], np.full(40, 127))
    assert np.array_equal(codes[7], np.rint(2.0 ** np.arange(40) / 2.0 ** 39 * 127))


# ---- ternary product --------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows, d, m, group, pad", [(1, 1, 1, 0, 0), (1, 96, 96, 64, 0), (2, 255, 17, 0, 1), (16, 257, 33, 128, 3), (17, 640, 100, 192, 0), (33, 1000, 130, 256, 5), (65, 513, 515, 320, 0),
                                                    (70, 2560, 200, 0, 16), (3, 4097, 48, 1024, 0), (300, 777, 391, 64, 1), (515, 1024, 640, 0, 0), (1000, 300, 1029, 512, 4)])
def test_matmul(ctx, kind, rows, d, m, group, pad):
    g = gen(rows + d + m)
    W = torch.randint(-1, 2, (d, m), generator=g).to(torch.int8)
    groups = -(-d // group) if group else 1
    w_scales = torch.rand(groups, m, generator=g) + 0.5
    codes = torch.randint(-128, 128, (rows, d), generator=g).to(torch.int8)
    scales = torch.rand(rows, generator=g) * 0.02
    weights = ctx.clear_weights_prepare(W.numpy(), w_scales.numpy(), group)
    out = strided(torch.zeros(rows, m, dtype=TYPES[kind]), pad)
    ctx.clear_matmul(weights, strided(codes, pad), scales.cuda(), out)
    size = group or d
    c = torch.nn.functional.pad(codes.double(), (0, groups * size - d)).reshape(rows, groups, size).transpose(0, 1)
    w = torch.nn.functional.pad(W.double(), (0, 0, 0, groups * size - d)).reshape(groups, size, m)
    parts = torch.bmm(c, w) * w_scales.double()[:, None]
    want = parts.sum(0) * scales.double()[:, None]
    # each group's sum is exact (parts of it, of 64 rows at least, where they are scaled apart), its product and every addition rounded in 32 bits, then by the rows' scale and once to the type
    terms = (c.abs() @ w.abs() * w_scales.double()[:, None]).sum(0) * scales.double()[:, None]
    off = (out.cpu().double() - want).abs()
    flushed = 2.0 ** -25 if kind == "f16" else 0  # half a step of the smallest numbers
    assert (off <= half_step(kind) * want.abs() * (1 + 1e-6) + (0 if not group else (d // 64 + 6)) * U32 * terms + 3 * U32 * want.abs() + flushed).all()
    weights.free()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows, d, m, group, pad", [(1500, 2048, 2050, 0, 0), (1300, 2000, 3001, 0, 5), (2050, 1030, 2500, 128, 0), (2000, 1536, 2600, 256, 16), (1111, 1543, 4100, 0, 0)])
def test_matmul_of_many_rows(ctx, kind, rows, d, m, group, pad):
    """Sizes where the matrix cores decide: rows that are aligned and that are not, edges in every direction."""
    test_matmul(ctx, kind, rows, d, m, group, pad)


def test_matmul_scales_pass_nan_and_rows_stay_apart(ctx):
    W = np.ones((64, 16), dtype=np.int8)
    weights = ctx.clear_weights_prepare(W, np.ones(16, dtype=np.float32))
    codes = torch.ones(3, 64, dtype=torch.int8, device="cuda")
    out = ctx.clear_matmul(weights, codes, torch.tensor([1.0, math.nan, 0.5], device="cuda"), dtype=torch.float32).cpu()
    assert (out[0] == 64).all() and out[1].isnan().all() and (out[2] == 32).all()
    weights.free()


def test_weights_that_are_not_ternary_are_refused(ctx):
    from paper_2509_09424_amd import EnsiError
    W = np.zeros((300, 20), dtype=np.int8)
    W[299, 19] = 2
    with pytest.raises(EnsiError, match="-1, 0 or 1"):
        ctx.clear_weights_prepare(W, np.ones(20, dtype=np.float32))


# ---- cache ------------------------------------------------------------------------------------------------------------------


def e4m3(codes):
    return codes.view(torch.float8_e4m3fn).float()


class Cache:
    """Sequences with `ctxs` cached and `news` new tokens on pages in random order; what no token has is NaN, codes and scales alike."""

    def __init__(self, ctx, ctxs, news, heads, dim, page, seed, powers=(-8, 3)):
        g = self.g = gen(seed)
        self.ctxs, self.news, self.heads, self.dim, self.page = ctxs, news, heads, dim, page
        need = [-(-(c + n) // page) for c, n in zip(ctxs, news)]
        width, pages = max(max(need), 1) + 1, sum(need) + 2
        order = torch.randperm(pages, generator=g)
        self.table = torch.full((len(ctxs), width), -1, dtype=torch.int32)
        at = 0
        for i, k in enumerate(need):
            self.table[i, :k] = order[at:at + k]
            at += k
        self.codes = {x: torch.full((pages, heads, page, dim), 0x7f, dtype=torch.uint8) for x in "kv"}
        self.scales = {x: torch.full((pages, heads, page // 16), math.nan) for x in "kv"}
        for i, c in enumerate(ctxs):
            self.fill(i, 0, c, powers)
        self.begin = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32)
        self.lengths = torch.tensor(ctxs, dtype=torch.int32)
        self.tokens = int(sum(news))

    def fill(self, i, a, b, powers):
        for x in "kv":
            for p in range(a, b):
                one, r = int(self.table[i, p // self.page]), p % self.page
                if r % 16 == 0 or p == a:
                    self.scales[x][one, :, r // 16] = 2.0 ** torch.randint(powers[0], powers[1], (self.heads,), generator=self.g).float()
                self.codes[x][one, :, r] = (torch.randn(self.heads, self.dim, generator=self.g) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

    def fill_new(self, powers=(-8, 3)):
        """New tokens as clear_append would have left them; whole blocks get a scale of their own."""
        for i, (c, n) in enumerate(zip(self.ctxs, self.news)):
            if c % 16:
                self.fill_codes(i, c, min(c + n, c + 16 - c % 16))
            self.fill(i, c + min(n, -c % 16), c + n, powers)

    def fill_codes(self, i, a, b):
        for x in "kv":
            for p in range(a, b):
                self.codes[x][int(self.table[i, p // self.page]), :, p % self.page] = (torch.randn(self.heads, self.dim, generator=self.g) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

    def wrap(self, ctx):
        self.dev = [t.clone().cuda() for t in (self.codes["k"], self.codes["v"], self.scales["k"], self.scales["v"])]
        self.where = [t.cuda() for t in (self.table, self.begin, self.lengths)]
        return ctx.clear_cache(*self.dev)

    def values(self, x, i, h):
        """Tokens of sequence i and head h in 64 bits."""
        n = self.ctxs[i] + self.news[i]
        p = torch.arange(n)
        one = self.table[i, p // self.page].long()
        return e4m3(self.codes[x][one, h, p % self.page]).double() * self.scales[x][one, h, p % self.page // 16].double()[:, None]


# ---- append -----------------------------------------------------------------------------------------------------------------


def turn32(x, cos, sin, rot, pairs):
    """Rotation in 32 bits, every product and sum rounded by itself."""
    x = x.float().numpy().copy()
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if pairs == "neighbours" else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., lo].copy(), x[..., hi].copy()
    x[..., lo], x[..., hi] = a * cos - b * sin, b * cos + a * sin
    return x


def append_reference(c, k, v, cos, sin, rot, pairs):
    """Codes and scales after the append, from the definition."""
    codes, scales = {x: t.clone() for x, t in c.codes.items()}, {x: t.clone() for x, t in c.scales.items()}
    for i, (ctx_len, new) in enumerate(zip(c.ctxs, c.news)):
        first, pos = int(c.begin[i]), np.arange(ctx_len, ctx_len + new)
        kk = turn32(k[first:first + new], cos[pos][:, None], sin[pos][:, None], rot, pairs) if rot else k[first:first + new].float().numpy()
        for x, t in (("k", kk), ("v", v[first:first + new].float().numpy())):
            for start in range(ctx_len - ctx_len % 16, ctx_len + new if new else 0, 16):
                one, r = int(c.table[i, start // c.page]), start % c.page
                a, b = max(ctx_len, start), min(ctx_len + new, start + 16)
                for h in range(c.heads):
                    part = t[a - ctx_len:b - ctx_len, h]
                    fine = np.isfinite(part)
                    most = np.abs(part[fine]).max() if fine.any() else 0.0
                    e = -64
                    while float(most) > 448 * 2.0 ** e:
                        e += 1
                    scale = 2.0 ** e
                    if a > start:
                        old = float(scales[x][one, h, r // 16])
                        if old < scale:
                            codes[x][one, h, r:r + a - start] = (e4m3(codes[x][one, h, r:r + a - start]) * (old / scale)).to(torch.float8_e4m3fn).view(torch.uint8)
                        scale = max(scale, old)
                    scales[x][one, h, r // 16] = scale
                    y = np.where(fine, part / np.float32(scale), np.float32(math.nan))
                    codes[x][one, h, r + a - start:r + b - start] = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, scales


def same_codes(got, want):
    """Equal as numbers: every NaN is the same, whatever its sign."""
    a, b = e4m3(got).nan_to_num(nan=1e9), e4m3(want).nan_to_num(nan=1e9)
    return torch.equal(a, b)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("ctxs, news, q_heads, heads, dim, rot, pairs, page", [
    ([0], [1], 1, 1, 64, 64, "half", 16), ([15, 16, 17, 0, 100], [1, 1, 1, 1, 1], 4, 2, 128, 128, "half", 64), ([0, 3, 40], [33, 0, 17], 3, 3, 96, 48, "neighbours", 16),
    ([7], [100], 8, 1, 256, 256, "neighbours", 32), ([1, 250], [31, 14], 2, 2, 192, 96, "half", 128), ([5, 9], [2, 300], 5, 5, 64, 32, "half", 48), ([12], [20], 2, 1, 128, 0, "half", 16)])
def test_append(ctx, kind, ctxs, news, q_heads, heads, dim, rot, pairs, page):
    c = Cache(ctx, ctxs, news, heads, dim, page, sum(ctxs) + dim)
    q = torch.randn(c.tokens, q_heads, dim, generator=c.g).to(TYPES[kind])
    both = torch.randn(c.tokens, 2 * heads, dim, generator=c.g) * 2.0 ** torch.randint(-6, 7, (c.tokens, 2 * heads, 1), generator=c.g).float()
    both = both.to(TYPES[kind])
    positions = max(a + b for a, b in zip(ctxs, news))
    angle = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(0, max(rot, 2), 2) / max(rot, 2))
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    codes, scales = append_reference(c, both[:, :heads], both[:, heads:], cos, sin, rot, pairs)
    cache, dev = c.wrap(ctx), both.cuda()
    q_out = strided(torch.zeros_like(q), 8)
    table, begin, lengths = c.where
    turn = (torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()) if rot else (None, None)
    got = ctx.clear_append(cache, table, begin, lengths, dev[:, :heads], dev[:, heads:], *turn, q=strided(q, 3), q_out=q_out, pairs=pairs, max_new=max(news))
    cache.check()
    assert got is q_out
    for x, (cd, sc) in zip("kv", ((c.dev[0], c.dev[2]), (c.dev[1], c.dev[3]))):
        assert same_codes(cd.cpu(), codes[x]) and torch.equal(sc.cpu().nan_to_num(nan=-1.0), scales[x].nan_to_num(nan=-1.0))
    where = np.concatenate([np.arange(a, a + n) for a, n in zip(ctxs, news)]).astype(int)
    if rot:
        want = torch.from_numpy(turn32(q, cos[where][:, None], sin[where][:, None], rot, pairs)).to(TYPES[kind])
    else:
        want = q
    assert torch.equal(q_out.cpu(), want)
    # the same into q itself, as one array of queries, keys and values
    cache.free()
    cache = c.wrap(ctx)
    qkv = torch.cat([q, both], 1).cuda()
    ctx.clear_append(cache, table, begin, lengths, qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:], *turn, q=qkv[:, :q_heads], q_out=qkv[:, :q_heads], pairs=pairs)
    assert torch.equal(qkv[:, :q_heads].cpu(), want) and torch.equal(qkv[:, q_heads:].cpu(), both) and same_codes(c.dev[1].cpu(), codes["v"])
    cache.check()
    cache.free()


def test_append_keeps_every_code_and_its_rounding(ctx):
    """All codes survive a larger scale as torch rounds them; values with infinities, NaN, zeros and the borders of the scale."""
    c = Cache(ctx, [8], [1], 1, 64, 16, 1, powers=(0, 1))
    one = int(c.table[0, 0])
    for x in "kv":
        c.codes[x][one, 0, :4] = torch.arange(256, dtype=torch.uint8).reshape(4, 64)
    for most, e in ((448.0, 0), (449.0, 1), (448.0 * 2, 1), (1e30, 91), (448 * 2.0 ** 40, 40), (0.0, 0)):
        k = torch.zeros(1, 1, 64)
        k[0, 0, 5], k[0, 0, 6], k[0, 0, 7], k[0, 0, 8] = most, math.inf, math.nan, -most / 3
        codes, scales = append_reference(c, k, k, None, None, 0, "half")
        assert float(scales["k"][one, 0, 0]) == 2.0 ** e
        cache = c.wrap(ctx)
        ctx.clear_append(cache, *c.where, k.cuda(), k.cuda(), None, None)
        for x, (cd, sc) in zip("kv", ((c.dev[0], c.dev[2]), (c.dev[1], c.dev[3]))):
            assert same_codes(cd.cpu(), codes[x]) and torch.equal(sc.cpu().nan_to_num(nan=-1.0), scales[x].nan_to_num(nan=-1.0))
        cache.free()


# ---- attention --------------------------------------------------------------------------------------------------------------


def attention_reference(c, q, cap, window, score, bias):
    """Outputs in 64 bits, and the sums of their terms' sizes, weights of unseen places and their values left out."""
    heads, group = c.heads, q.shape[1] // c.heads
    out, size, top = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
    for i, (ctx_len, new) in enumerate(zip(c.ctxs, c.news)):
        first = int(c.begin[i])
        for h in range(heads):
            k, v = c.values("k", i, h), c.values("v", i, h)
            for t in range(new):
                hi = ctx_len + t + 1
                lo = max(0, hi - window) if window else 0
                for j in range(h * group, (h + 1) * group):
                    s = k[lo:hi] @ q[first + t, j].double() / math.sqrt(c.dim)
                    top[first + t, j] = s.abs().max()
                    if cap:
                        s = cap * torch.tanh(s / cap)
                    p = torch.softmax(s, 0) if score == "softmax" else torch.sigmoid(s + bias)
                    out[first + t, j], size[first + t, j] = p @ v[lo:hi], p @ v[lo:hi].abs()
    return out, size, top


def attention_near(c, kind, got, q, cap=0.0, window=0, score="softmax", bias=0.0):
    out, size, top = attention_reference(c, q, cap, window, score, bias)
    # scores: a sum of dim products in 32 bits (dim steps of the largest part at most, here relative to 3 deviations of random signs), the exponent's argument rounded at its own size; weights
    # rounded to 11 bits (bf16) or 22 (f16), and by 2^-25 of the largest contribution where they are small; the sum over the keys in 32 bits
    n = max(a + b for a, b in zip(c.ctxs, c.news))
    weight = (2.0 ** -11 if kind == "bf16" else 2.0 ** -21) + n * U32 + (top[..., None] * 8 + 16 + (4 * cap if cap else 0)) * 2 * U32
    largest = torch.stack([c.values("v", i, h)[:a + b].nan_to_num().abs().max() for i, (a, b) in enumerate(zip(c.ctxs, c.news)) if b for h in range(c.heads)]).max()
    peak = size.amax(2, keepdim=True)
    bound = half_step(kind) * out.abs() * (1 + 2.0 ** -7) + weight * size + n * 2.0 ** -25 * peak * 64 + torch.finfo(TYPES[kind]).smallest_normal * 2.0 ** -7
    off = (got.cpu().double() - out).abs()
    assert largest > 0 and (off <= bound).all(), (off / bound).max()


CASES = [
    # ctxs, news, heads, group, dim, page, cap, window, score
    ([0], [1], 1, 1, 64, 16, 0.0, 0, "softmax"),
    ([31, 0, 500], [1, 1, 1], 2, 4, 128, 64, 0.0, 0, "softmax"),
    ([1000, 77, 16, 15], [1, 1, 1, 1], 1, 8, 96, 16, 30.0, 100, "softmax"),
    ([300], [1], 5, 3, 256, 128, 0.0, 17, "sigmoid"),
    ([0, 20, 130], [50, 0, 7], 2, 1, 96, 16, 20.0, 33, "sigmoid"),
    ([5], [130], 1, 5, 128, 48, 0.0, 0, "softmax"),
    ([64, 3], [40, 90], 2, 2, 64, 32, 5.0, 1, "softmax"),
    ([100], [70], 1, 2, 192, 16, 0.0, 50, "softmax"),
    ([2500], [3], 1, 20, 128, 64, 0.0, 0, "softmax"),
    ([33], [300], 1, 1, 256, 64, 0.0, 200, "softmax"),
    ([200, 0], [150, 260], 1, 4, 64, 16, 0.0, 0, "sigmoid"),
]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("ctxs, news, heads, group, dim, page, cap, window, score", CASES)
def test_attention(ctx, kind, ctxs, news, heads, group, dim, page, cap, window, score):
    c = Cache(ctx, ctxs, news, heads, dim, page, sum(ctxs) + sum(news) + dim)
    c.fill_new()
    q = (torch.randn(c.tokens, heads * group, dim, generator=c.g) / 16).to(TYPES[kind])
    cache = c.wrap(ctx)
    out = strided(torch.full_like(q, 9.0), 5)
    bias = -math.log(max(ctxs) + max(news)) if score == "sigmoid" else 0.0
    ctx.clear_attention(cache, *c.where, strided(q, 3), out, cap=cap, window=window, score=score, bias=bias, max_new=max(news), max_length=max(a + b for a, b in zip(ctxs, news)))
    cache.check()
    attention_near(c, kind, out, q, cap, window, score, bias)
    # the bounds that a caller gives do not change what is computed, only how it is split
    again = ctx.clear_attention(cache, *c.where, strided(q, 3), None, cap=cap, window=window, score=score, bias=bias)
    attention_near(c, kind, again, q, cap, window, score, bias)
    cache.free()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("ctxs, news, heads, group, dim, page, cap, window, score", [
    ([70, 0], [1800, 1000], 8, 4, 64, 16, 0.0, 0, "softmax"), ([200], [1500], 8, 4, 128, 64, 0.0, 0, "softmax"), ([33], [1501], 8, 2, 96, 32, 20.0, 300, "softmax"),
    ([10], [1500], 4, 6, 192, 16, 0.0, 0, "sigmoid"), ([100], [1450], 8, 4, 256, 64, 0.0, 500, "softmax"), ([5, 300, 40], [1500, 0, 911], 8, 2, 64, 48, 9.0, 0, "sigmoid")])
def test_attention_of_prompts(ctx, kind, ctxs, news, heads, group, dim, page, cap, window, score):
    """Prompts that share their keys in a workgroup; the reference on the GPU in 64 bits, a head at a time."""
    c = Cache(ctx, ctxs, news, heads, dim, page, sum(ctxs) + sum(news) + dim)
    c.fill_new()
    q = (torch.randn(c.tokens, heads * group, dim, generator=c.g) / 16).to(TYPES[kind])
    cache = c.wrap(ctx)
    bias = -math.log(max(ctxs) + max(news)) if score == "sigmoid" else 0.0
    got = ctx.clear_attention(cache, *c.where, q.cuda(), cap=cap, window=window, score=score, bias=bias, max_new=max(news), max_length=max(a + b for a, b in zip(ctxs, news)))
    cache.check()
    for i, (ctx_len, new) in enumerate(zip(ctxs, news)):
        first, n = int(c.begin[i]), ctx_len + new
        at = torch.arange(ctx_len, n, device="cuda")[:, None]
        key = torch.arange(n, device="cuda")
        seen = (key <= at) & (key > at - window if window else key >= 0)
        for h in range(heads if new else 0):
            k, v = c.values("k", i, h).cuda(), c.values("v", i, h).cuda()
            for j in range(h * group, (h + 1) * group):
                s = q[first:first + new, j].cuda().double() @ k.T / math.sqrt(dim)
                top = s.abs().amax(1, keepdim=True)
                if cap:
                    s = cap * torch.tanh(s / cap)
                p = torch.softmax(s.masked_fill(~seen, -math.inf), 1) if score == "softmax" else torch.sigmoid(s + bias).masked_fill(~seen, 0)
                out, size = p @ v, p @ v.abs()
                # as in attention_near, with weights of 11 bits in either type: their roundings, each half a step at most, add up to no more than half a step of the sum of sizes
                weight = 2.0 ** -11 + n * U32 + (top * 8 + 16 + 4 * cap) * 2 * U32
                bound = half_step(kind) * out.abs() * (1 + 2.0 ** -7) + weight * size + n * 2.0 ** -25 * size.amax(1, keepdim=True) * 64 + torch.finfo(TYPES[kind]).smallest_normal * 2.0 ** -7
                off = (got[first:first + new, j].double() - out).abs()
                assert (off <= bound).all(), (i, j, (off / bound).max())
    cache.free()


@pytest.mark.parametrize("news", [[1], [90], [400]])
def test_attention_with_scales_far_apart(ctx, news):
    """Value scales from 2^-60 to 2^100 in one sequence: the tokens that a row leans on decide, and what is small beside them is lost only beside them."""
    c = Cache(ctx, [200], news, 1, 64, 16, 3)
    c.fill_new()
    for b in range((200 + news[0]) // 16 + 1):
        one, r = int(c.table[0, b * 16 // 16]), 0
        c.scales["v"][one, 0, r] = 2.0 ** (-60 if b % 2 else -30)
    c.scales["v"][int(c.table[0, 2]), 0, 0] = 2.0 ** 100
    q = (torch.randn(c.tokens, 2, 64, generator=c.g) / 16).to(torch.bfloat16)
    cache = c.wrap(ctx)
    got = ctx.clear_attention(cache, *c.where, q.cuda())
    attention_near(c, "bf16", got, q)
    # a window past the large block: only the small ones count
    got = ctx.clear_attention(cache, *c.where, q.cuda(), window=100)
    attention_near(c, "bf16", got, q, window=100)
    cache.free()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("window", [0, 700])
def test_attention_of_prompts_with_nan_and_scales_far_apart(ctx, score, window):
    """A long prompt whose keys are shared in workgroups: a NaN among the values of one head reaches its place in the rows that see it, one among another's keys the whole
    rows that see it; a third head's value scales are far apart."""
    c = Cache(ctx, [50], [1800], 8, 64, 16, 7)
    c.fill_new()
    page = lambda p: int(c.table[0, p // 16])  # noqa: E731
    for b in range(1850 // 16 + 1):
        c.scales["v"][page(16 * b), 5, 0] = 2.0 ** (-60 if b % 2 else -30)
    c.scales["v"][page(900), 5, 0] = 2.0 ** 100
    q = (torch.randn(c.tokens, 32, 64, generator=c.g) / 16).to(torch.bfloat16)
    call = lambda: ctx.clear_attention(c.wrap(ctx), *c.where, q.cuda(), window=window, score=score).cpu()  # noqa: E731
    clean = call()
    assert clean.isfinite().all()
    at_v, at_k = 777, 1001
    c.codes["v"][page(at_v), 2, at_v % 16, 11] = 0xff
    c.codes["k"][page(at_k), 6, at_k % 16, 3] = 0x7f
    got = call()
    pos = torch.arange(50, 1850)
    sees = lambda p: (pos >= p) & (pos - window < p if window else pos >= 0)  # noqa: E731
    want = clean.clone()
    want[sees(at_v), 8:12, 11] = math.nan
    want[sees(at_k), 24:28] = math.nan
    assert torch.equal(got.isnan(), want.isnan())
    # (its code counts as 0 where it is not seen, and the other heads are as they were)
    assert torch.equal(got.nan_to_num(), want.nan_to_num())
    # the head with scales far apart, against the definition
    k, v = c.values("k", 0, 5).cuda(), c.values("v", 0, 5).cuda()
    key, at = torch.arange(1850, device="cuda"), pos.cuda()[:, None]
    seen = (key <= at) & (key > at - window if window else key >= 0)
    for j in range(20, 24):
        s = q[:, j].cuda().double() @ k.T / 8
        p = torch.softmax(s.masked_fill(~seen, -math.inf), 1) if score == "softmax" else torch.sigmoid(s).masked_fill(~seen, 0)
        out, size = p @ v, p @ v.abs()
        bound = half_step("bf16") * out.abs() * 1.01 + (2.0 ** -11 + 1850 * U32 + (s.abs().amax(1, keepdim=True) * 8 + 16) * 2 * U32) * size + 1850 * 2.0 ** -25 * size.amax(1, keepdim=True) * 64 + 2.0 ** -133
        off = (got[:, j].cuda().double() - out).abs()
        assert (off <= bound).all(), (off / bound).max()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("news, window", [([40], 0), ([40], 12), ([1], 30), ([300], 0), ([300], 64)])
def test_attention_and_nan_in_the_cache(ctx, score, news, window):
    """A NaN among the values reaches the rows that see its token, in its place only; a NaN among the keys the whole rows that see it."""
    c = Cache(ctx, [50], news, 1, 64, 16, 5)
    c.fill_new()
    n = 50 + news[0]
    q = (torch.randn(c.tokens, 2, 64, generator=c.g) / 16).to(torch.float16)
    at_v, at_k = n - 15, n - 9
    clean = ctx.clear_attention(c.wrap(ctx), *c.where, q.cuda(), window=window, score=score).cpu()
    one = int(c.table[0, at_v // 16])
    c.codes["v"][one, 0, at_v % 16, 11] = 0xff
    got = ctx.clear_attention(c.wrap(ctx), *c.where, q.cuda(), window=window, score=score).cpu()
    for t in range(news[0]):
        p = 50 + t
        seen = p >= at_v and (not window or p - window < at_v)
        want = clean[t].clone()
        if seen:
            want[:, 11] = math.nan
        assert torch.equal(got[t].isnan(), want.isnan()) and torch.equal(got[t].nan_to_num(), want.nan_to_num()), t
    c.codes["v"][one, 0, at_v % 16, 11] = 0
    c.codes["k"][int(c.table[0, at_k // 16]), 0, at_k % 16, 3] = 0x7f
    got = ctx.clear_attention(c.wrap(ctx), *c.where, q.cuda(), window=window, score=score).cpu()
    for t in range(news[0]):
        p = 50 + t
        assert got[t].isnan().all() if p >= at_k and (not window or p - window < at_k) else not got[t].isnan().any(), t


def test_what_does_not_fit_is_left_out_and_reported(ctx):
    """Bad pages and lengths on the device: no access outside the cache, the other sequences are served, the check says so once."""
    from paper_2509_09424_amd import EnsiError
    ctxs, news = [40, 40, 40], [1, 1, 1]
    c = Cache(ctx, ctxs, news, 1, 64, 16, 6)
    c.fill_new()
    q = (torch.randn(3, 2, 64, generator=c.g) / 16).to(torch.bfloat16)
    kv = torch.randn(3, 2, 64, generator=c.g).to(torch.bfloat16).cuda()
    good = ctx.clear_attention(c.wrap(ctx), *c.where, q.cuda()).cpu()
    for what in ("page", "negative page", "length", "begin", "new", "past"):
        cache = c.wrap(ctx)
        table, begin, lengths = (t.clone() for t in c.where)
        more = {}
        if what == "page":
            table[1] = 1 << 30
        elif what == "negative page":
            table[1] = -5
        elif what == "length":
            lengths[1] = 1 << 30
        elif what == "begin":
            begin[:] = torch.tensor([0, 1, 5, -1])
        elif what == "new":
            begin[:] = torch.tensor([0, 1, 3, 3])
            more = {"max_new": 1}
        else:
            lengths[1] = -1
        before = [t.clone() for t in c.dev]
        ctx.clear_append(cache, table, begin, lengths, kv[:, :1], kv[:, 1:], None, None, **more)
        with pytest.raises(EnsiError, match="left out"):
            cache.check()
        cache.check()
        wrote = [(a != b).flatten(1).any(1) for a, b in zip((t.nan_to_num(nan=-1.0) if t.is_floating_point() else t for t in before), (t.nan_to_num(nan=-1.0) if t.is_floating_point() else t for t in c.dev))]
        assert not any(w[int(c.table[1, 2])] for w in wrote)
        cache = c.wrap(ctx)
        out = torch.full_like(q, 3.0).cuda()
        ctx.clear_attention(cache, table, begin, lengths, q.cuda(), out, **more)
        with pytest.raises(EnsiError, match="left out"):
            cache.check()
        out = out.cpu()
        assert torch.equal(out[0], good[0])
        if "page" in what:
            assert (out[1] == 0).all() and torch.equal(out[2], good[2])
        elif what in ("length", "past"):
            assert (out[1] == 3).all() and torch.equal(out[2], good[2])
        cache.free()


def test_empty_calls(ctx):
    c = Cache(ctx, [4], [0], 1, 64, 16, 6)
    cache = c.wrap(ctx)
    none = torch.zeros(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    ctx.clear_append(cache, *c.where, none, none, None, None)
    assert ctx.clear_attention(cache, *c.where, none).shape == none.shape
    codes, scales = ctx.clear_norm(none[:, 0], torch.ones(64, dtype=torch.bfloat16, device="cuda"))
    weights = ctx.clear_weights_prepare(np.ones((64, 16), dtype=np.int8), np.ones(16, dtype=np.float32))
    assert ctx.clear_matmul(weights, codes, scales, dtype=torch.float32).shape == (0, 16)
    weights.free()
    cache.check()
    cache.free()


# ---- offsets past 32 bits ---------------------------------------------------------------------------------------------------


def test_product_and_norm_past_32_bits(ctx):
    """Codes, outputs and sums with more than 2^31 elements: the last rows are what a call of these rows alone gives."""
    rows, d, m, last = 70000, 32768, 32000, 600
    x = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
    x[-last:] = torch.randn(last, d, generator=gen(1)).to(torch.bfloat16).cuda()
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(x)
    codes, scales = ctx.clear_norm(x, gain, out=out, codes=torch.empty(rows, d, dtype=torch.int8, device="cuda"))
    few_out = torch.empty_like(x[-last:])
    few_codes, few_scales = ctx.clear_norm(x[-last:], gain, out=few_out, codes=torch.empty(last, d, dtype=torch.int8, device="cuda"))
    near = 64 * U32  # of each from the sum of squares, as in test_norm
    assert torch.equal(codes[-last:], few_codes) and not codes[:-last].any() and not scales[:-last].any()
    assert ((scales[-last:].double() - few_scales.double()).abs() <= 2 * near * few_scales.double()).all()
    assert ((out[-last:].double() - few_out.double()).abs() <= (2 * near + 2 * half_step("bf16")) * few_out.double().abs() * (1 + 2.0 ** -7)).all()
    del x, out
    W = torch.randint(-1, 2, (64, m), generator=gen(2)).to(torch.int8)
    weights = ctx.clear_weights_prepare(W.numpy(), np.full(m, 0.5, dtype=np.float32))
    narrow = codes[:, -64:]  # rows of 64 codes, 32768 apart
    scales = torch.ones(rows, device="cuda")
    got = ctx.clear_matmul(weights, narrow, scales, dtype=torch.bfloat16)
    few = ctx.clear_matmul(weights, few_codes[:, -64:], scales[:last], dtype=torch.bfloat16)
    want = few_codes[:, -64:].double() @ W.cuda().double() * 0.5
    assert torch.equal(got[-last:], few) and torch.equal(few, want.to(torch.bfloat16)) and not got[:-last].any()
    weights.free()


@pytest.mark.parametrize("news", [[1], [3], [900]])
def test_pages_past_32_bits(ctx, news):
    """A cache of 4.6 GiB for keys and as much for values, pages at its end, held as e4m3: the codes and outputs of a small one of bytes, bit for bit."""
    heads, dim, page = 8, 128, 64
    c = Cache(ctx, [200], news, heads, dim, page, 21)
    q = (torch.randn(c.tokens, 2 * heads, dim, generator=c.g) / 16).to(torch.bfloat16).cuda()
    kv = [torch.randn(c.tokens, heads, dim, generator=c.g).to(torch.bfloat16).cuda() for _ in "kv"]
    small = c.wrap(ctx)
    pages, mine = 75000, len(c.codes["k"])
    far = pages - mine
    big = [torch.zeros(pages, heads, page, dim, dtype=torch.uint8, device="cuda") for _ in "kv"] + [torch.ones(pages, heads, page // 16, device="cuda") for _ in "kv"]
    for b, t in zip(big, c.dev):
        b[far:] = t
    large = ctx.clear_cache(*(b.view(torch.float8_e4m3fn) for b in big[:2]), *big[2:])
    table, begin, lengths = c.where
    results = []
    for cache, where in ((small, table), (large, torch.where(table < 0, table, table + far))):
        ctx.clear_append(cache, where, begin, lengths, *kv, None, None)
        results.append(ctx.clear_attention(cache, where, begin, lengths, q, max_new=news[0], max_length=200 + news[0]))
        cache.check()
    for b, t in zip(big, c.dev):
        assert torch.equal(b[far:].view(torch.uint8), t.view(torch.uint8))
        assert (b[:far] == (1 if b.is_floating_point() else 0)).all()
    assert torch.equal(*results)
    small.free()
    large.free()


def test_most_rows_and_largest_bounds(ctx):
    """The most rows of a product and of a norm, and the largest bounds that a caller may give: the results of ordinary calls."""
    rows = 1 << 20
    W = torch.randint(-1, 2, (70, 16), generator=gen(3)).to(torch.int8)
    weights = ctx.clear_weights_prepare(W.numpy(), np.full(16, 0.5, dtype=np.float32))
    codes = torch.randint(-128, 128, (rows, 70), generator=gen(4)).to(torch.int8).cuda()
    got = ctx.clear_matmul(weights, codes, torch.ones(rows, device="cuda"), dtype=torch.float32)
    assert torch.equal(got, (codes.float() @ W.cuda().float()) * 0.5)  # sums of whole numbers up to 70 x 128: exact
    weights.free()
    x = torch.ones(2 * rows, 9, dtype=torch.bfloat16, device="cuda")
    codes, scales = ctx.clear_norm(x, x[0], codes=torch.zeros(2 * rows, 9, dtype=torch.int8, device="cuda"))
    assert (codes == 127).all() and (scales == scales[0]).all()
    c = Cache(ctx, [40, 3], [20, 1], 1, 64, 16, 22)
    q = (torch.randn(c.tokens, 2, 64, generator=c.g) / 16).to(torch.bfloat16)
    kv = torch.randn(c.tokens, 2, 64, generator=c.g).to(torch.bfloat16).cuda()
    results = []
    for bounds in ((20, 60), (1 << 20, 1 << 30)):
        cache = c.wrap(ctx)
        ctx.clear_append(cache, *c.where, kv[:, :1], kv[:, 1:], None, None, max_new=bounds[0])
        got = ctx.clear_attention(cache, *c.where, q.cuda(), max_new=bounds[0], max_length=bounds[1])
        cache.check()
        results.append([t.nan_to_num(nan=-1.0) if t.is_floating_point() else t for t in c.dev])
        c.codes, c.scales = {"k": c.dev[0].cpu(), "v": c.dev[1].cpu()}, {"k": c.dev[2].cpu(), "v": c.dev[3].cpu()}
        attention_near(c, "bf16", got, q)
        cache.free()
    assert all(torch.equal(a, b) for a, b in zip(*results))


# ---- streams and graphs -----------------------------------------------------------------------------------------------------


def test_current_stream_and_graph(ctx):
    """A decoding step on a stream of its own and in a graph, replayed with other inputs and with eager work between: the eager results, every time."""
    c = Cache(ctx, [700, 3], [1, 1], 2, 64, 16, 8)
    g = c.g
    weights = ctx.clear_weights_prepare(torch.randint(-1, 2, (256, 512), generator=g).to(torch.int8).numpy(), np.full(512, 0.01, dtype=np.float32))
    gain = torch.ones(256, device="cuda", dtype=torch.bfloat16)
    cos, sin = torch.rand(800, 32, device="cuda"), torch.rand(800, 32, device="cuda")
    x, r = torch.zeros(2, 256, device="cuda", dtype=torch.bfloat16), torch.zeros(2, 256, device="cuda", dtype=torch.bfloat16)
    cache = c.wrap(ctx)
    start = [t.clone() for t in c.dev]
    table, begin, lengths = c.where
    codes, scales = torch.empty(2, 256, dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
    qkv, out = torch.empty(2, 512, device="cuda", dtype=torch.bfloat16), torch.empty(2, 4, 64, device="cuda", dtype=torch.bfloat16)

    def step():
        ctx.clear_norm(x, gain, residual=r, sum_out=r, codes=codes, scales=scales)
        ctx.clear_matmul(weights, codes, scales, qkv)
        heads = qkv.view(2, 8, 64)
        q = ctx.clear_append(cache, table, begin, lengths, heads[:, 4:6], heads[:, 6:], cos, sin, q=heads[:, :4], q_out=heads[:, :4], max_new=1)
        ctx.clear_attention(cache, table, begin, lengths, q, out, max_new=1, max_length=800)

    def begin_with(seed):
        for t, s in zip(c.dev, start):
            t.copy_(s)
        x.copy_(torch.randn(2, 256, generator=gen(seed)))
        r.zero_()

    wants = []
    for seed in range(4):
        begin_with(seed)
        step()
        wants.append([out.clone(), r.clone()] + [t.clone() for t in c.dev[:2]])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        begin_with(1)
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, wants[1][0])
    begin_with(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        for seed in range(4):
            begin_with(seed)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip([out, r] + c.dev[:2], wants[seed])), (turn, seed)
            begin_with(seed + 7)
            step()  # eager work between the replays
    cache.check()
    weights.free()
    cache.free()
