"""The operators of a decoder layer on clear activations, as measurable cases: the layer that the encrypted path computes, with
the same ternary weights, for requests that are not encrypted, for the ranges that scales and levels are chosen by, and for what
is compared with a decrypted result.

norm       h = x + residual in the tensors' type; codes = round(p 127 / max |p|) with p = h gain, and one scale a row,
           max |p| / (127 sqrt(mean h^2 + eps)).  The root cancels in the codes, so that they are whole numbers defined by products
           of 32 bits alone: they are returned as such, beside their scales.
matmul     out[t][i] = scale_t sum_g w_gi sum_{j in group g} W[j][i] codes[t][j], W in {-1, 0, 1}.
append     queries and keys rotated by their positions; keys and values stored as e4m3 in a paged cache, one power of two as scale for
           each block of 16 tokens and head.  Returned: the rotated queries and the whole updated cache.
attention  of the last `new` tokens of each sequence over that cache: grouped heads, causal, with a window, a cap on the scores,
           and the softmax or the paper's sigmoid in its place.

Inputs are made on the GPU; lengths of sequences follow from the case, so that its work does.
"""
import math

import torch

own = False

BLOCK = 16  # tokens that share a scale in the cache
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one token of a decoder of width 2560 between two layers: latency decides
        {"name": "norm_token", "op": "norm", "rows": 1, "d": 2560, "pad": 0, "type": "bf16", "residual": True, "full": False},
        # a prompt of 4096 tokens at the same width, the codes that its projections multiply
        {"name": "norm_prompt", "op": "norm", "rows": 4096, "d": 2560, "pad": 0, "type": "bf16", "residual": True, "full": False},
        # the norm ahead of a wide down projection in an odd width, rows that do not start on 16 bytes, values kept as well
        {"name": "norm_odd", "op": "norm", "rows": 517, "d": 6911, "pad": 3, "type": "f16", "residual": False, "full": True},
        # one token through the up projection of a feed-forward block
        {"name": "matmul_token", "op": "matmul", "rows": 1, "d": 2560, "m": 6912, "group": 0, "type": "bf16"},
        # a batch of decoding sequences through the down projection, weights with a scale for every 128 rows
        {"name": "matmul_batch", "op": "matmul", "rows": 37, "d": 6912, "m": 2560, "group": 128, "type": "f16"},
        # a prompt through the up projection: the matrix cores decide
        {"name": "matmul_prompt", "op": "matmul", "rows": 4096, "d": 2560, "m": 6912, "group": 0, "type": "bf16"},
        # a decoding step of 64 sequences: one token each
        {"name": "append_step", "op": "append", "seqs": 64, "new": 1, "ctx": 1000, "q_heads": 20, "kv_heads": 5, "dim": 128, "rot": 128, "pairs": "half", "page": 64, "type": "bf16"},
        # prompts of up to 2048 tokens, 16 heads of 96, the layout of neighbouring pairs that the paper's RoPE has
        {"name": "append_prompt", "op": "append", "seqs": 4, "new": 2048, "ctx": 0, "q_heads": 16, "kv_heads": 16, "dim": 96, "rot": 96, "pairs": "neighbours", "page": 16, "type": "f16"},
        # the next token of one long document
        {"name": "attention_long", "op": "attention", "seqs": 1, "new": 1, "ctx": 32767, "q_heads": 20, "kv_heads": 5, "dim": 128, "page": 64, "type": "bf16", "score": "softmax", "cap": 0.0, "window": 0},
        # a decoding step of 48 sequences of all lengths up to 8192
        {"name": "attention_batch", "op": "attention", "seqs": 48, "new": 1, "ctx": 8191, "q_heads": 20, "kv_heads": 5, "dim": 128, "page": 64, "type": "bf16", "score": "softmax", "cap": 0.0, "window": 0},
        # the second part of a long prompt, behind 2048 tokens that the cache holds
        {"name": "attention_prompt", "op": "attention", "seqs": 1, "new": 4096, "ctx": 2048, "q_heads": 20, "kv_heads": 5, "dim": 128, "page": 64, "type": "bf16", "score": "softmax", "cap": 0.0, "window": 0},
        # short prompts under sigmoid attention with a cap and a window, in the paper's head width
        {"name": "attention_sigmoid", "op": "attention", "seqs": 5, "new": 77, "ctx": 1500, "q_heads": 16, "kv_heads": 16, "dim": 96, "page": 16, "type": "f16", "score": "sigmoid", "cap": 30.0, "window": 640},
    ]


def _between(rng, low, high):
    """A whole number from low to high, spread over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5)))))))


def draw(rng):
    op = rng.choice(("norm", "matmul", "append", "attention"))
    if op == "norm":
        d = _between(rng, 64, 8192)
        return {"op": op, "rows": _between(rng, 1, max(1, min(4096, 4096 * 2560 // d))), "d": d, "pad": rng.choice((0, 0, 1, 8)),
                "type": rng.choice(("f32", "bf16", "f16")), "residual": rng.random() < 0.6, "full": rng.random() < 0.4}
    if op == "matmul":
        d, m = _between(rng, 96, 8192), _between(rng, 96, 8192)
        return {"op": op, "rows": _between(rng, 1, max(1, min(4096, 4096 * 2560 * 6912 // (d * m)))), "d": d, "m": m,
                "group": rng.choice((0, 0, 64, 128, 256)), "type": rng.choice(("f32", "bf16", "f16"))}
    dim = rng.choice((64, 96, 128, 256))
    kv = rng.choice((1, 2, 4, 5, 8, 16))
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 5, 8) if g * kv <= 40])
    page = rng.choice((16, 32, 64, 128))
    if op == "append":
        new = 1 if rng.random() < 0.4 else _between(rng, 2, 2048)
        seqs = _between(rng, 1, 64 if new == 1 else max(1, 4096 // new))
        return {"op": op, "seqs": seqs, "new": new, "ctx": _between(rng, 1, 1024) - 1, "q_heads": heads, "kv_heads": kv, "dim": dim,
                "rot": rng.choice((dim, dim // 2)), "pairs": rng.choice(("half", "neighbours")), "page": page, "type": rng.choice(("f32", "bf16", "f16"))}
    if rng.random() < 0.6:
        new, ctx = 1, _between(rng, 16, 32768) - 1
        seqs = _between(rng, 1, max(1, min(64, 200000 // (ctx + 1), 200000 * 5 * 128 // ((ctx + 1) * kv * dim))))
    else:
        new, ctx, seqs = _between(rng, 2, 2048), _between(rng, 1, 2048) - 1, rng.choice((1, 2, 3))
        while seqs * new * (ctx + new) * heads * dim > 4096 * 4096 * 20 * 128:
            new = max(2, new // 2)
    return {"op": op, "seqs": seqs, "new": new, "ctx": ctx, "q_heads": heads, "kv_heads": kv, "dim": dim, "page": page, "type": rng.choice(("bf16", "bf16", "f16")),
            "score": rng.choice(("softmax", "softmax", "sigmoid")), "cap": rng.choice((0.0, 0.0, 30.0)), "window": rng.choice((0, 0, _between(rng, 16, 4096)))}


def _lengths(case):
    """(tokens in the cache, new tokens) of each sequence: the first has the most, the others all lengths below."""
    part = lambda most, i, step: most if i == 0 else int(most * ((i * step) % 1.0))  # noqa: E731
    return [(part(case["ctx"], i, 0.6180339887), 1 if case["new"] == 1 else part(case["new"], i, 0.7548776662)) for i in range(case["seqs"])]


def _pairs_seen(case):
    """Sum over the new tokens of the keys that each attends to."""
    w = case["window"]
    total = 0
    for ctx, new in _lengths(case):
        for p in range(ctx + 1, ctx + new + 1):
            total += min(p, w) if w else p
    return total


def work(case):
    size = SIZE[case["type"]]
    if case["op"] == "norm":
        n = case["rows"] * case["d"]
        return {"bytes": n * size * (1 + 2 * case["residual"] + case["full"]) + n + 4 * case["rows"] + size * case["d"], "flops": 4 * n}
    if case["op"] == "matmul":
        rows, d, m = case["rows"], case["d"], case["m"]
        groups = -(-d // case["group"]) if case["group"] else 1
        return {"bytes": d * m / 4 + 4 * groups * m + rows * (d + 4) + size * rows * m, "flops": 2 * rows * d * m}
    hq, hk, dim = case["q_heads"], case["kv_heads"], case["dim"]
    new = sum(n for _, n in _lengths(case))
    if case["op"] == "append":
        return {"bytes": new * dim * (2 * hq * size + 2 * hk * (size + 1)) + new * 4 * case["rot"], "flops": 3 * new * case["rot"] * (hq + hk)}
    w = case["window"]
    keys = sum(min(ctx + n, w + n - 1) if w else ctx + n for ctx, n in _lengths(case) if n)
    return {"bytes": keys * hk * (2 * dim + 8 / BLOCK) + 2 * new * hq * dim * size, "flops": 4 * _pairs_seen(case) * hq * dim}


# ---- inputs -----------------------------------------------------------------------------------------------------------------

_context = None


def _ctx():
    """The library's context: one for the program's life, at the smallest ring in use."""
    global _context
    if _context is None:
        from paper_2509_09424_amd import Context
        _context = Context(12, 36, 3, 37, 1, 1, 30)
    return _context


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = TYPES[case["type"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": case}
    if case["op"] == "norm":
        rows, d, wide = case["rows"], case["d"], case["d"] + case["pad"]
        s["x"] = normal(rows, wide).to(kind)[:, :d]
        if case["residual"]:
            s["residual"] = (normal(rows, wide) * 3).to(kind)[:, :d]
        s["gain"] = (1 + 0.2 * normal(d)).to(kind)
    elif case["op"] == "matmul":
        rows, d, m = case["rows"], case["d"], case["m"]
        groups = -(-d // case["group"]) if case["group"] else 1
        u = torch.rand(d, m, generator=g, device="cuda")
        s["W"] = (u >= 0.7).to(torch.int8) - (u < 0.3).to(torch.int8)
        s["w_scales"] = torch.rand(groups, m, generator=g, device="cuda") * 0.02 + 0.01
        s["codes"] = (normal(rows, d) * 32).round().clamp(-127, 127).to(torch.int8)
        s["scales"] = torch.rand(rows, generator=g, device="cuda") * 0.02 + 0.01
    else:
        lengths = _lengths(case)
        page, hk, dim = case["page"], case["kv_heads"], case["dim"]
        width = max(-(-(c + n) // page) for c, n in lengths)
        pages = sum(-(-(c + n) // page) for c, n in lengths) + 3
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros(len(lengths), width, dtype=torch.int32, device="cuda")
        at = 0
        for i, (c, n) in enumerate(lengths):
            k = -(-(c + n) // page)
            table[i, :k] = order[at:at + k]
            at += k
        s["table"], s["spare"] = table, order[-1:]  # a page that no sequence has
        starts = [0]
        for _, n in lengths:
            starts.append(starts[-1] + n)
        s["begin"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["lengths"] = torch.tensor([c for c, _ in lengths], dtype=torch.int32, device="cuda")
        new = starts[-1]
        for name in ("k", "v"):
            old = torch.empty(pages, hk, page, dim, dtype=torch.uint8, device="cuda")
            for p in range(0, pages, 256):  # in parts: the cache alone has to fit
                q = min(pages, p + 256)
                old[p:q] = (normal(q - p, hk, page, dim) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            s[name + "_cache"] = old
            s[name + "_scale"] = torch.exp2(torch.randint(-7, -5, (pages, hk, page // BLOCK), generator=g, device="cuda").float())
        s["q"] = normal(new, case["q_heads"], dim).to(kind)
        if case["op"] == "append":
            both = normal(new, 2 * hk, dim).to(kind)  # keys and values as the projection leaves them, side by side
            s["k"], s["v"] = both[:, :hk], both[:, hk:]
            angle = torch.arange(case["ctx"] + case["new"], dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (
                -torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kind = TYPES[case["type"]]
    if case["op"] == "norm":
        s["sum"] = torch.empty(case["rows"], case["d"], dtype=kind, device="cuda")
        s["codes"] = torch.empty(case["rows"], case["d"], dtype=torch.int8, device="cuda")
        s["scales"] = torch.empty(case["rows"], device="cuda")
        s["full"] = torch.empty(case["rows"], case["d"], dtype=kind, device="cuda")
    elif case["op"] == "matmul":
        s["out"] = torch.empty(case["rows"], case["m"], dtype=kind, device="cuda")
        if own:
            s["weights"] = _ctx().clear_weights_prepare(s.pop("W").cpu().numpy(), s.pop("w_scales").cpu().numpy(), case["group"])
        else:
            s["W"] = s["W"].float()
    else:
        s["out"] = torch.empty_like(s["q"])
        if own:
            s["cache"] = _ctx().clear_cache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    return s


def run(s):
    case = s["case"]
    return {"norm": _norm, "matmul": _matmul, "append": _append, "attention": _attention}[case["op"]](s, case)


# ---- norm -------------------------------------------------------------------------------------------------------------------


def _norm(s, case):
    x, gain, residual = s["x"], s["gain"], s.get("residual")
    if own:
        _ctx().clear_norm(x, gain, residual=residual, eps=EPS, sum_out=s["sum"] if residual is not None else None, out=s["full"] if case["full"] else None,
                          codes=s["codes"], scales=s["scales"])
        got = {"codes": s["codes"], "scales": s["scales"]}
        if residual is not None:
            got["sum"] = s["sum"]
        if case["full"]:
            got["full"] = s["full"]
        return got
    got = {}
    h = x
    if residual is not None:
        h = got["sum"] = (x.float() + residual.float()).to(x.dtype)
    h = h.float()
    root = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    p = h * gain.float()
    most = p.abs().amax(1, keepdim=True)
    got["codes"] = torch.round(p * (127.0 / most)).to(torch.int8)
    got["scales"] = (root * (most / 127.0))[:, 0]
    if case["full"]:
        got["full"] = (p * root).to(x.dtype)
    return got


# ---- matmul -----------------------------------------------------------------------------------------------------------------


def _matmul(s, case):
    if own:
        _ctx().clear_matmul(s["weights"], s["codes"], s["scales"], s["out"])
        return s["out"]
    codes, W = s["codes"].float(), s["W"]
    rows, d, m, size = case["rows"], case["d"], case["m"], case["group"]
    if not size:
        y = codes @ W * s["w_scales"]
    else:
        groups = -(-d // size)
        codes = torch.nn.functional.pad(codes, (0, groups * size - d)).reshape(rows, groups, size).transpose(0, 1).contiguous()
        W = torch.nn.functional.pad(W, (0, 0, 0, groups * size - d)).reshape(groups, size, m)
        y = (torch.bmm(codes, W) * s["w_scales"][:, None, :]).sum(0)
    return (y * s["scales"][:, None]).to(TYPES[case["type"]])


# ---- append -----------------------------------------------------------------------------------------------------------------


def _places(s, count):
    """Of each new token: its sequence and its position."""
    t = torch.arange(count, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["begin"], t, right=True) - 1
    return seq, s["lengths"][seq] + t - s["begin"][seq]


def _rotate(x, cos, sin, rot, pairs):
    x = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs == "neighbours" else (x[..., :rot // 2], x[..., rot // 2:rot])
    a0, b0 = a.clone(), b.clone()
    a.copy_(a0 * cos - b0 * sin)
    b.copy_(b0 * cos + a0 * sin)
    return x


def _power(most):
    """The smallest power of two by which `most` becomes at most 448, not below 2^-64."""
    part, e = torch.frexp(most.double() / 448.0)
    return torch.exp2((e - (part == 0.5).to(e.dtype)).clamp(min=-64).double()).float()


def _append(s, case):
    kc, vc, ks, vs = s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]
    if own:
        _ctx().clear_append(s["cache"], s["table"], s["begin"], s["lengths"], s["k"], s["v"], s["cos"], s["sin"], q=s["q"], q_out=s["out"],
                            pairs=case["pairs"], max_new=case["new"])
    else:
        page, hk, count, seqs = case["page"], case["kv_heads"], s["q"].shape[0], case["seqs"]
        seq, pos = _places(s, count)
        cos, sin = s["cos"][pos][:, None, :], s["sin"][pos][:, None, :]
        s["out"] = _rotate(s["q"].float(), cos, sin, case["rot"], case["pairs"]).to(s["q"].dtype)
        where = s["table"][seq, pos // page].long()
        block = where * (page // BLOCK) + pos % page // BLOCK
        # the blocks that held tokens before, one a sequence: their 16 places
        had = (s["lengths"] % BLOCK != 0) & (s["begin"][1:] > s["begin"][:-1])
        first = s["lengths"] - s["lengths"] % BLOCK
        last_page = torch.where(had, s["table"].gather(1, (first // page).clamp(max=s["table"].shape[1] - 1).long()[:, None])[:, 0], s["spare"]).long()
        block_had = last_page * (page // BLOCK) + first % page // BLOCK  # of the spare page where there is none
        line = (first % page)[:, None] + torch.arange(BLOCK, device="cuda")
        is_old = (had[:, None] & (torch.arange(BLOCK, device="cuda") < (s["lengths"] % BLOCK)[:, None]))[:, :, None, None]
        for codes, scales, x in ((kc, ks, _rotate(s["k"].float(), cos, sin, case["rot"], case["pairs"])), (vc, vs, s["v"].float())):
            flat = scales.transpose(1, 2).reshape(-1, hk)
            most = torch.zeros_like(flat).scatter_reduce(0, block[:, None].expand(-1, hk), x.abs().amax(2), "amax")
            touched = torch.zeros(len(flat), 1, dtype=torch.bool, device="cuda").index_fill_(0, block, True)
            kept = torch.zeros(len(flat), 1, device="cuda").index_add_(0, block_had, had.float()[:, None]) > 0
            new = torch.where(touched, torch.maximum(_power(most), torch.where(kept, flat, torch.zeros_like(flat))), flat)
            scales.copy_(new.reshape(-1, page // BLOCK, hk).transpose(1, 2))
            before = codes[last_page[:, None], :, line]
            again = (before.view(torch.float8_e4m3fn).float() * (flat / new)[block_had][:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            # sequences without an older part write the spare page's lines back as they are
            codes[last_page[:, None], :, line] = torch.where(is_old, again, before)
            codes[where, :, pos % page] = (x / new[block][:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return {"q": s["out"], "k": kc.view(torch.float8_e4m3fn), "v": vc.view(torch.float8_e4m3fn), "k_scale": ks, "v_scale": vs}


# ---- attention --------------------------------------------------------------------------------------------------------------


def _bias(case):
    return -math.log(case["ctx"] + case["new"])  # sigmoid weights of about one in all


def _values(codes, scales, table):
    """Every sequence's cache as numbers: [sequences, heads, tokens, width]."""
    x = codes[table.long()].view(torch.float8_e4m3fn).float()
    x = x.unflatten(3, (-1, BLOCK)) * scales[table.long()][..., None, None]
    return x.flatten(3, 4).transpose(1, 2).flatten(2, 3)


def _attention(s, case):
    if own:
        _ctx().clear_attention(s["cache"], s["table"], s["begin"], s["lengths"], s["q"], s["out"], cap=case["cap"], window=case["window"], score=case["score"],
                               bias=_bias(case), max_new=case["new"], max_length=case["ctx"] + case["new"])
        return s["out"]
    hq, hk, dim, new, seqs = case["q_heads"], case["kv_heads"], case["dim"], case["new"], case["seqs"]
    seq, pos = _places(s, s["q"].shape[0])
    i = pos - s["lengths"][seq]
    q = torch.zeros(seqs, new, hq, dim, device="cuda")
    q[seq, i] = s["q"].float()
    q = q.reshape(seqs, new, hk, hq // hk, dim).permute(0, 2, 3, 1, 4).reshape(seqs * hk, -1, dim)
    k = _values(s["k_cache"], s["k_scale"], s["table"])
    t = torch.bmm(q, k.flatten(0, 1).transpose(1, 2)).reshape(seqs, hk, hq // hk, new, -1).mul_(dim ** -0.5)
    del k
    if case["cap"]:
        t = torch.tanh(t.div_(case["cap"])).mul_(case["cap"])
    at = (s["lengths"][:, None] + torch.arange(new, device="cuda"))[:, None, None, :, None]
    key = torch.arange(t.shape[-1], device="cuda")
    seen = key <= at
    if case["window"]:
        seen = seen & (key > at - case["window"])
    if case["score"] == "sigmoid":
        p = torch.sigmoid(t + _bias(case)).masked_fill_(~seen, 0.0)
    else:
        t = t.masked_fill_(~seen, -torch.inf)
        p = torch.exp(t - t.amax(-1, keepdim=True))
        p = p.div_(p.sum(-1, keepdim=True))
    del t
    v = _values(s["v_cache"], s["v_scale"], s["table"])
    o = torch.bmm(p.reshape(seqs * hk, -1, p.shape[-1]), v.flatten(0, 1))
    o = o.reshape(seqs, hk, hq // hk, new, dim).permute(0, 3, 1, 2, 4).reshape(seqs, new, hq, dim)
    return o[seq, i].to(s["q"].dtype)


# ---- the same from the definitions, in 64 bits ------------------------------------------------------------------------------


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        got = {}
        h = s["x"]
        if case["residual"]:
            h = got["sum"] = (h.double() + s["residual"].double()).to(h.dtype)  # its rounding belongs to the definition
        p = h.double() * s["gain"].double()
        root = 1 / torch.sqrt((h.double() ** 2).sum(1) / case["d"] + EPS)
        got |= {"codes": None, "scales": root * p.abs().max(1).values / 127}
        if case["full"]:
            got["full"] = p * root[:, None]
        return got
    if case["op"] == "matmul":
        W, size = s["W"].double(), case["group"] or case["d"]
        W = W * s["w_scales"].double().repeat_interleave(size, 0)[:case["d"]]
        return s["scales"].double()[:, None] * (s["codes"].double() @ W)
    if case["op"] == "append":
        return _exact_append(s, case)
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    group, page, at = case["q_heads"] // case["kv_heads"], case["page"], 0
    for i, (ctx, new) in enumerate(_lengths(case)):
        if not new:
            continue
        n = ctx + new
        pages = s["table"][i, :-(-n // page)].long()
        low = max(0, ctx - case["window"] + 1) if case["window"] else 0
        place = torch.arange(low, n, device="cuda")
        for h in range(case["kv_heads"]):
            k, v = ((s[x + "_cache"][pages[place // page], h, place % page].view(torch.float8_e4m3fn).double()
                     * s[x + "_scale"][pages[place // page], h, place % page // BLOCK].double()[:, None]) for x in "kv")
            for j in range(h * group, (h + 1) * group):
                t = s["q"][at:at + new, j].double() @ k.T / math.sqrt(case["dim"])
                if case["cap"]:
                    t = case["cap"] * torch.tanh(t / case["cap"])
                back = torch.arange(ctx, n, device="cuda")[:, None] - place
                dark = (back < 0) | (back >= case["window"] if case["window"] else torch.zeros_like(back, dtype=torch.bool))
                if case["score"] == "sigmoid":
                    p = (1 / (1 + torch.exp(-(t + _bias(case))))).masked_fill(dark, 0)
                else:
                    p = torch.softmax(t.masked_fill(dark, -torch.inf), 1)
                out[at:at + new, j] = p @ v
        at += new
    return out


def _exact_append(s, case):
    page, half, at = case["page"], case["rot"] // 2, 0
    if case["pairs"] == "neighbours":
        low, high = torch.arange(half, device="cuda") * 2, torch.arange(half, device="cuda") * 2 + 1
    else:
        low, high = torch.arange(half, device="cuda"), torch.arange(half, device="cuda") + half
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    scales = {n: s[n + "_scale"].double() for n in "kv"}
    codes = {n: s[n + "_cache"].view(torch.float8_e4m3fn).double() for n in "kv"}
    for i, (ctx, new) in enumerate(_lengths(case)):
        turn = torch.complex(s["cos"][ctx:ctx + new].double(), s["sin"][ctx:ctx + new].double())[:, None]
        for x in (q, k):
            z = torch.complex(x[at:at + new][..., low], x[at:at + new][..., high]) * turn
            x[at:at + new, :, low], x[at:at + new, :, high] = z.real, z.imag
        for start in range(ctx - ctx % BLOCK, ctx + new if new else 0, BLOCK):
            one, r = int(s["table"][i, start // page]), start % page
            a, b = max(ctx, start), min(ctx + new, start + BLOCK)
            for n, x in (("k", k), ("v", v)):
                part = x[at + a - ctx:at + b - ctx].transpose(0, 1)
                most = part.abs().amax((1, 2))
                e = torch.ceil(torch.log2(most / 448)).clamp(min=-64)
                was, now = scales[n][one, :, r // BLOCK].clone(), torch.exp2(e)
                if a > start:
                    now = torch.maximum(now, was)
                    codes[n][one, :, r:r + a - start] = (codes[n][one, :, r:r + a - start] * (was / now)[:, None, None]).to(torch.float8_e4m3fn).double()
                scales[n][one, :, r // BLOCK] = now
                codes[n][one, :, r + a - start:r + b - start] = (part / now[:, None, None]).to(torch.float8_e4m3fn).double()
        at += new
    return {"q": q, "k": codes["k"], "v": codes["v"], "k_scale": scales["k"], "v_scale": scales["v"]}
