"""The operators of token mixing that are measured: heads of queries and keys, a cache in 4 bits, attention over it.

A row is the channel vector of one token.  Three kinds of case:

  heads    queries and keys of a row, each head normed by itself and rotated by the token's position, in one pass
  append   keys (normed and rotated) and values written into a paged cache that holds them in 4 bits, and what it then holds for them
  attend   attention of rows of queries over the cache of their stream

and four ways in which tokens come:

  rows     consecutive rows, each with a position of its own
  each     one new token for each of many streams (serving)
  map      the flagged pixels of a batch of maps: a list of pixel indices with its length on the GPU; a stream is one map
  prompt   several tokens of several streams, the last ones of each

The cache holds 32 values of a head as 4-bit floating-point codes (sign, two bits of exponent, one of mantissa: 0, 0.5, 1,
1.5, 2, 3, 4, 6) with one power of two for a scale, the smallest that keeps the largest of them within 6; values go to the
nearest code, ties to the even one.  codes is [pages, 2 (keys, values), heads, page, dim / 2] bytes, the even value in the
low half, scales [pages, 2, heads, page, dim / 32] bytes, exponents with a bias of 127.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
MAX_FLOPS, MAX_BYTES, MAX_SCORES = 5.8e11, 3.0e8, 3.0e9  # what a drawn case may cost


def listed():
    return [
        # queries and keys of one token: latency
        _heads("heads_one_token", how="rows", rows=1, q_heads=32, heads=8, dim=128, dtype="f16", norm="rms", rot=128, style="halves"),
        # odd numbers, a norm with a mean, part of a head rotated by pairs of neighbours
        _heads("heads_ragged", how="rows", rows=1021, q_heads=9, heads=3, dim=96, dtype="f32", norm="layer", rot=64, style="pairs"),
        # every token of a long batch
        _heads("heads_long_batch", how="rows", rows=16384, q_heads=32, heads=8, dim=128, dtype="bf16", norm="rms", rot=128, style="halves"),
        # a decode step of a serving batch: one token a stream
        _append("append_one_each", how="each", streams=64, length=4096, tokens=1, heads=8, dim=128, dtype="bf16", norm="rms", rot=128, style="halves", page=64),
        # the flagged pixels of 64 streams of 64x64 at 10 % density, rotated by row and column
        _append("append_flagged_pixels", how="map", streams=64, length=4096, tokens=0, heads=8, dim=64, dtype="f16", norm="rms", rot=64, style="halves", page=64, density=0.1),
        # prompts of several streams, small pages
        _append("append_prompt", how="prompt", streams=5, length=4099, tokens=4099, heads=8, dim=128, dtype="bf16", norm="none", rot=128, style="halves", page=16),
        # one token of one stream: latency
        _attend("attend_one_token", how="each", streams=1, length=1000, tokens=1, q_heads=32, heads=8, dim=128, dtype="f16", page=64),
        # a decode step of a serving batch, streams of all lengths
        _attend("attend_one_each", how="each", streams=64, length=8192, tokens=1, q_heads=32, heads=8, dim=128, dtype="bf16", page=64),
        # one token behind a very long text
        _attend("attend_long_cache", how="each", streams=1, length=262143, tokens=1, q_heads=32, heads=8, dim=128, dtype="f16", page=64),
        # odd numbers, a window, fp32
        _attend("attend_ragged", how="prompt", streams=7, length=1531, tokens=37, q_heads=9, heads=3, dim=96, dtype="f32", page=16, window=200),
        # flagged pixels against all pixels of their map
        _attend("attend_flagged_pixels", how="map", streams=64, length=4096, tokens=0, q_heads=8, heads=8, dim=64, dtype="f16", page=64, density=0.1),
        # whole prompts of several streams
        _attend("attend_prompt", how="prompt", streams=3, length=6000, tokens=6000, q_heads=32, heads=8, dim=128, dtype="bf16", page=64),
    ]


def _heads(name, how, rows, q_heads, heads, dim, dtype, norm, rot, style, streams=0, length=0, density=0.0):
    return dict(name=name, op="heads", how=how, rows=rows, streams=streams, length=length, density=density, q_heads=q_heads, heads=heads, dim=dim,
                dtype=dtype, norm=norm, rot=rot, style=style)


def _append(name, how, streams, length, tokens, heads, dim, dtype, norm, rot, style, page, density=0.0):
    return dict(name=name, op="append", how=how, streams=streams, length=length, tokens=tokens, density=density, heads=heads, dim=dim, dtype=dtype, norm=norm,
                rot=rot, style=style, page=page)


def _attend(name, how, streams, length, tokens, q_heads, heads, dim, dtype, page, window=0, density=0.0):
    return dict(name=name, op="attend", how=how, streams=streams, length=length, tokens=tokens, density=density, q_heads=q_heads, heads=heads, dim=dim,
                dtype=dtype, page=page, window=window)


def draw(rng):
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        op, dtype, dim = rng.choice(["heads", "append", "attend"]), rng.choice(["f32", "f16", "bf16"]), rng.choice([32, 64, 96, 128, 128, 192, 256])
        heads = rng.choice([1, 2, 3, 4, 5, 8, 8, 16])
        q_heads = heads * rng.choice([1, 1, 2, 3, 4, 4, 7, 8])
        norm, rot, style = rng.choice(["none", "rms", "rms", "layer"]), rng.choice([0, dim, dim, dim // 32 * 16]), rng.choice(["halves", "pairs"])
        page, density = rng.choice([16, 32, 64, 128]), rng.choice([0.03, 0.1, 0.3])
        how = rng.choice(["rows", "map"] if op == "heads" else ["each", "map", "prompt"])
        if how == "map":
            side = rng.randint(8, 64)
            streams, length, tokens = rng.randint(1, 64), side * side, 0
        elif how == "each":
            streams, length, tokens = spread(1, 128), spread(1, 200000), 1
        else:
            streams, length = rng.randint(1, 9), spread(2, 6000)
            tokens = spread(1, length)
        if op == "heads":
            rows = spread(1, 16384)
            if how == "rows":
                streams, length, density = 0, 0, 0.0
            else:
                rows = 0
            case = _heads("", how, rows, q_heads, heads, dim, dtype, norm, rot, style, streams, length, density)
        elif op == "append":
            case = _append("", how, streams, length, tokens, heads, dim, dtype, norm, rot, style, page, density if how == "map" else 0.0)
        else:
            window = 0 if how == "map" else rng.choice([0, 0, spread(1, length)])
            case = _attend("", how, streams, length, tokens, q_heads, heads, dim, dtype, page, window, density if how == "map" else 0.0)
        w = work(case)
        cache = 0 if op == "heads" else streams * length * heads * dim
        scores = 0 if op != "attend" else streams * q_heads * max(_counts(case)) * (1.5 if how == "map" else 1.0) * length
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and cache <= MAX_BYTES and scores <= MAX_SCORES:
            return {k: v for k, v in case.items() if k != "name"}


# ---- which tokens ---------------------------------------------------------------------------------------------------
def _lengths(case):
    """Tokens of each stream: all lengths from a short one to the whole."""
    n, streams = case["length"], case["streams"]
    if case["how"] == "map":
        return [n] * streams
    low = n // 16 if case["how"] == "each" else n // 2
    return [max(1, n - (s * 7919 % 101) * (n - low) // 101) for s in range(streams)]


def _counts(case):
    """Rows of each stream."""
    if case["how"] == "map":
        return [max(1, round(case["length"] * case["density"]))] * case["streams"]  # (on average)
    return [min(case["tokens"], n) for n in _lengths(case)]


def _rows_of(case):
    return case["rows"] if case["how"] == "rows" else sum(_counts(case))


def _keys(case):
    """Pairs of a row and a key of it, and keys that some row wants."""
    pairs = wanted = 0
    for n, rows in zip(_lengths(case), _counts(case)):
        if case["how"] == "map":
            pairs, wanted = pairs + rows * n, wanted + n
            continue
        reach = case["window"] if case["window"] else n
        first, last = n - rows + 1, n                   # keys up to the first and the last row
        full = max(0, last - max(first, reach) + 1)     # rows with a whole window
        part = rows - full
        pairs += full * reach + part * (first + first + part - 1) // 2
        wanted += min(n, rows + reach - 1)
    return pairs, wanted


def _tokens(case, gen, s):
    """The rows' tokens as a program keeps them, and what the plain forms make of them: `stream` and `pos` of each row, `most` rows a stream."""
    how = case["how"]
    s.update(idx=None, count=None, streams=None, positions=None, lens=None, most=1)
    if how == "map":
        streams, n = case["streams"], case["length"]
        s["m"] = m = _rows_of(case)
        s["idx"] = torch.zeros(streams * n, dtype=torch.int32, device="cuda")
        s["idx"][:m] = torch.randperm(streams * n, device="cuda", generator=gen)[:m].sort().values
        s["count"] = torch.tensor([m], dtype=torch.int32, device="cuda")
        s["most"] = int(torch.bincount(s["idx"][:m] // n).max())
        return
    if how == "rows":
        s["m"] = case["rows"]
        s["positions"] = torch.randint(0, s["table_rows"], (s["m"],), dtype=torch.int32, device="cuda", generator=gen)
        return
    lens, counts = torch.tensor(_lengths(case)), torch.tensor(_counts(case))
    s["m"], s["most"] = int(counts.sum()), int(counts.max())
    at = torch.repeat_interleave(torch.arange(len(lens)), counts)
    rank = torch.arange(s["m"]) - (counts.cumsum(0) - counts)[at]
    s["lens"] = lens.to(torch.int32).cuda()
    s["positions"] = (lens[at] - counts[at] + rank).to(torch.int32).cuda()
    if how == "prompt":
        s["streams"] = at.to(torch.int32).cuda()


def _table(case):
    """cos and sin of each position's angles, [positions, rot / 2, 2]; on a map half of the pairs turn by the row and half by the column."""
    rot, n = case["rot"], case["length"] if case["how"] != "rows" else 32768
    if rot == 0:
        return None
    p = torch.arange(n, device="cuda", dtype=torch.float64)[:, None]
    if case["how"] == "map":
        side, quarter = math.isqrt(n), rot // 4
        f = 100.0 ** (-torch.arange(quarter, device="cuda", dtype=torch.float64) / quarter)
        a = torch.cat([torch.div(p, side, rounding_mode="floor") * f, torch.remainder(p, side) * f], 1)
    else:
        a = p * 10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) / (rot // 2))
    return torch.stack([torch.cos(a), torch.sin(a)], 2).float()


def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _norm(case, gen):
    if case["norm"] == "none":
        return None
    about = lambda mean: (mean + 0.1 * _normal(gen, case["dim"])).to(DTYPES[case["dtype"]])  # noqa: E731
    return case["norm"], about(1.0), about(0.0) if case["norm"] == "layer" else None


def _cache(case, gen, filled, s):
    """A cache whose pages lie in any order; maps have theirs one behind the other, and no table."""
    page, streams, heads, dim = case["page"], case["streams"], case["heads"], case["dim"]
    per_stream = -(-case["length"] // page)
    num = streams * per_stream
    s["pages"] = None if case["how"] == "map" else torch.randperm(num, device="cuda", generator=gen).to(torch.int32).view(streams, per_stream)
    s["codes"] = torch.zeros(num, 2, heads, page, dim // 2, dtype=torch.uint8, device="cuda")
    s["scales"] = torch.zeros(num, 2, heads, page, dim // 32, dtype=torch.uint8, device="cuda")
    if filled:
        by_channel = torch.exp(0.3 * _normal(gen, heads, 1, dim))
        step = max(1, (1 << 25) // (heads * page * dim))
        for at in range(0, num, step):
            for which in (0, 1):
                v = _normal(gen, min(step, num - at), heads, page, dim) * by_channel
                s["codes"][at:at + step, which], s["scales"][at:at + step, which] = _quantised(v)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s, dt, dim = {"case": case}, DTYPES[case["dtype"]], case["dim"]
    if case["op"] != "attend":
        s["table"] = _table(case)
        s["table_rows"] = 32768 if s["table"] is None else s["table"].shape[0]
    _tokens(case, gen, s)
    m, kv = s["m"], case["heads"] * dim
    if case["op"] == "heads":
        q = case["q_heads"] * dim
        s["x"] = (_normal(gen, m, q + 2 * kv) * torch.exp(0.3 * _normal(gen, q + 2 * kv))).to(dt)  # queries, keys and values of one product
        s["q"], s["k"] = s["x"][:, :q], s["x"][:, q:q + kv]
        s["q_norm"], s["k_norm"] = _norm(case, gen), _norm(case, gen)
    elif case["op"] == "append":
        x = (_normal(gen, m, 2 * kv) * torch.exp(0.3 * _normal(gen, 2 * kv))).to(dt)
        s["k"], s["v"], s["k_norm"] = x[:, :kv], x[:, kv:], _norm(case, gen)
        _cache(case, gen, False, s)
    else:
        s["q"] = (1.5 * _normal(gen, m, case["q_heads"] * dim)).to(dt)
        _cache(case, gen, True, s)
    if own:
        import paper_2203_03996_amd as pkg
        s["ctx"] = ctx = pkg.Context(0)
        if case["op"] != "attend":
            s["q_norm"], s["k_norm"] = (s.get(n) and pkg.RowNorm(*s[n], eps=EPS) for n in ("q_norm", "k_norm"))
            s["rotation"] = None if s["table"] is None else pkg.Rotation(s["table"], case["style"])
        if case["op"] != "heads":
            s["cache"] = pkg.TokenCache(ctx, case["streams"], case["length"], case["heads"], dim, dtype=dt, page=case["page"], pages=s["pages"],
                                        codes=s["codes"], scales=s["scales"])
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _row_tokens(s):
    """(stream, position) of each row."""
    if s["idx"] is not None:
        at = s["idx"][:s["m"]].long()
        return torch.div(at, s["case"]["length"], rounding_mode="floor"), at % s["case"]["length"]
    stream = torch.arange(s["m"], device="cuda") if s["streams"] is None else s["streams"].long()
    return stream, s["positions"].long()


def _turned(s, x, norm, dt):
    """Heads [rows, heads, dim] of x, normed and rotated, in the type `dt`."""
    case = s["case"]
    v = x.reshape(x.shape[0], -1, case["dim"]).to(dt)
    if norm is not None:
        kind, w, b = norm
        if kind == "layer":
            v = v - v.mean(2, keepdim=True)
        v = v / torch.sqrt((v * v).mean(2, keepdim=True) + EPS) * w.to(dt)
        if b is not None:
            v = v + b.to(dt)
    rot = case["rot"]
    if rot:
        cos, sin = s["table"][_row_tokens(s)[1]].to(dt).unbind(2)
        cos, sin = cos[:, None], sin[:, None]
        if case["style"] == "halves":
            a, b = v[..., :rot // 2], v[..., rot // 2:rot]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], 2)
        else:
            a, b = v[..., 0:rot:2], v[..., 1:rot:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], 3).flatten(2)
        v = torch.cat([turned, v[..., rot:]], 2)
    return v


def _quantised(v):
    """(codes, scales) of the last dimension of v."""
    blocks = v.unflatten(-1, (-1, 32))
    mantissa, exponent = torch.frexp(blocks.abs().amax(-1))
    e = (exponent - 2 - (mantissa <= 0.75).to(torch.int32)).clamp(-126, 127)
    u = torch.ldexp(blocks, -e[..., None])
    a = u.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0) + 8 * (u < 0).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _values(codes, scales):
    """The numbers, in 32 bits, that codes [..., dim / 2] and scales [..., dim / 32] stand for."""
    known = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device="cuda")
    v = torch.stack([known[(codes & 15).int()], known[(codes >> 4).int()]], -1).flatten(-2)
    power = torch.ldexp(torch.ones((), device="cuda"), scales.int() - 127)
    return (v.unflatten(-1, (-1, 32)) * power[..., None]).flatten(-2)


def _page_of(s, stream, block):
    per_stream = -(-s["case"]["length"] // s["case"]["page"])
    return stream * per_stream + block if s["pages"] is None else s["pages"][stream, block].long()


def _plain_append(s):
    case, dt = s["case"], DTYPES[s["case"]["dtype"]]
    stream, pos = _row_tokens(s)
    page, slot = _page_of(s, stream, torch.div(pos, case["page"], rounding_mode="floor")), pos % case["page"]
    # in 64 bits: a value next to the border of two codes
    k = _turned(s, s["k"], s["k_norm"], torch.float64)
    v = s["v"].reshape(s["m"], -1, case["dim"]).double()
    codes, scales = _quantised(torch.stack([k, v], 1))
    s["codes"][page, :, :, slot] = codes
    s["scales"][page, :, :, slot] = scales
    held = _values(s["codes"][page, :, :, slot], s["scales"][page, :, :, slot]).to(dt)
    return held[:, 0].flatten(1), held[:, 1].flatten(1)


def _plain_attend(s):
    case, dt, m = s["case"], DTYPES[s["case"]["dtype"]], s["m"]
    streams, n, heads, dim, most = case["streams"], case["length"], case["heads"], case["dim"], s["most"]
    stream, pos = _row_tokens(s)
    # the cache of every stream, [streams, heads, tokens, dim]
    blocks = torch.arange(-(-n // case["page"]), device="cuda")
    page = _page_of(s, torch.arange(streams, device="cuda")[:, None], blocks[None])
    kv = _values(s["codes"][page], s["scales"][page]).permute(2, 0, 3, 1, 4, 5).flatten(3, 4)[:, :, :, :n]
    # its rows, [streams, rows, ...]: those of a stream lie together
    rank = torch.arange(m, device="cuda") - torch.searchsorted(stream, stream)
    q = torch.zeros(streams, most, heads, case["q_heads"] // heads, dim, device="cuda")
    q[stream, rank] = s["q"].float().view(m, heads, -1, dim)
    low, high = (torch.zeros(streams, most, dtype=torch.long, device="cuda") for _ in range(2))
    if case["how"] == "map":
        high[stream, rank] = n
    else:
        high[stream, rank] = torch.minimum(pos + 1, s["lens"][stream].long())
        if case["window"]:
            low[stream, rank] = (pos + 1 - case["window"]).clamp(min=0)
    at = torch.arange(n, device="cuda")
    hidden = (at < low[..., None]) | (at >= high[..., None])
    w = torch.matmul(q.permute(0, 2, 3, 1, 4).flatten(2, 3), kv[0].transpose(2, 3)).unflatten(2, (-1, most)).mul_(1.0 / math.sqrt(dim))
    w.masked_fill_(hidden[:, None, None], -math.inf)
    w = w.sub_(w.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    out = torch.matmul(w.flatten(2, 3), kv[1]).unflatten(2, (-1, most)) / w.sum(-1, keepdim=True).clamp(min=1e-30)
    return out.permute(0, 3, 1, 2, 4)[stream, rank].flatten(1).to(dt)


def run(s):
    case = s["case"]
    if own:
        tokens = dict(idx=s["idx"], count=s["count"], positions=s["positions"])
        if case["op"] == "heads":
            q, k = s["ctx"].rows_heads(s["q"], s["k"], dim=case["dim"], q_norm=s["q_norm"], k_norm=s["k_norm"], rotation=s["rotation"], **tokens)
            return q[:s["m"]], k[:s["m"]]
        tokens["streams"] = s["streams"]
        if case["op"] == "append":
            s["cache"].append(s["k"], s["v"], norm=s["k_norm"], rotation=s["rotation"], **tokens)
            k, v = s["cache"].read(**tokens)
            return k[:s["m"]], v[:s["m"]]
        return s["cache"].attend(s["q"], lens=s["lens"], causal=case["how"] != "map", window=case["window"], **tokens)[:s["m"]]
    if case["op"] == "heads":
        dt = DTYPES[case["dtype"]]
        return tuple(_turned(s, x, norm, torch.float32).flatten(1).to(dt) for x, norm in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"])))
    return _plain_append(s) if case["op"] == "append" else _plain_attend(s)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------
def _exact_heads(s, x, norm):
    """By complex numbers: a pair turned by an angle is one multiplied with cos + i sin."""
    case, rows = s["case"], x.shape[0]
    d, rot = case["dim"], case["rot"]
    v = x.to(torch.float64).reshape(rows, -1, d)
    if norm is not None:
        kind, w, b = norm
        centre = v.sum(2, keepdim=True) / d if kind == "layer" else torch.zeros_like(v[..., :1])
        spread = (v - centre).square().sum(2, keepdim=True) / d + EPS
        v = (v - centre) * spread.rsqrt() * w.double() + (0.0 if b is None else b.double())
    if rot:
        pos = (s["idx"][:s["m"]] % case["length"] if s["idx"] is not None else s["positions"]).long()
        turn = torch.view_as_complex(s["table"].double())[pos][:, None]
        inner = v[..., :rot]
        pairs = inner.reshape(rows, -1, 2, rot // 2).transpose(2, 3) if case["style"] == "halves" else inner.reshape(rows, -1, rot // 2, 2)
        turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        turned = turned.transpose(2, 3).reshape(inner.shape) if case["style"] == "halves" else turned.reshape(inner.shape)
        v = torch.cat((turned, v[..., rot:]), dim=2)
    return v.reshape(rows, -1)


def _exact_held(v, d):
    """Rows of heads as a cache in 4 bits holds them: multiples of a step that doubles from 2 and from 4 on, rounded half to even."""
    b = v.reshape(v.shape[0], -1, 32)
    top = b.abs().max(2, keepdim=True).values
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top / 6.0, torch.ones_like(top)))))
    scale = torch.where(scale * 6.0 < top, scale * 2.0, torch.where(scale * 3.0 >= top, scale / 2.0, scale))  # (should a logarithm have rounded)
    u = b / scale
    step = 0.5 * torch.where(u.abs() < 2.0, 1.0, torch.where(u.abs() < 4.0, 2.0, 4.0).to(torch.float64))
    return (torch.round(u / step) * step * scale).reshape(v.shape)


def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    d, m = case["dim"], s["m"]
    if case["op"] == "heads":
        return _exact_heads(s, s["q"], s["q_norm"]), _exact_heads(s, s["k"], s["k_norm"])
    if case["op"] == "append":
        return _exact_held(_exact_heads(s, s["k"], s["k_norm"]), d), _exact_held(s["v"].double(), d)
    heads, group, n = case["heads"], case["q_heads"] // case["heads"], case["length"]
    out = torch.zeros(m, case["q_heads"], d, dtype=torch.float64, device="cuda")
    rows = torch.arange(m, device="cuda")
    stream = s["idx"][:m].long() // n if s["idx"] is not None else rows if s["streams"] is None else s["streams"].long()
    per_stream = -(-n // case["page"])
    held = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    for i in range(case["streams"]):
        mine = rows[stream == i]
        pages = torch.arange(i * per_stream, (i + 1) * per_stream, device="cuda") if s["pages"] is None else s["pages"][i].long()
        last = n if s["lens"] is None else _lengths(case)[i]
        t = torch.arange(last, device="cuda")
        if case["how"] == "map":
            seen = torch.ones(len(mine), last, dtype=torch.bool, device="cuda")
        else:
            p = s["positions"][mine].long()[:, None]
            seen = t <= p
            if case["window"]:
                seen &= t > p - case["window"]
        for h in range(heads):
            kv = []
            for which in (0, 1):
                byte = s["codes"][pages, which, h].reshape(-1, d // 2)[:last]
                nibble = torch.stack((byte & 0xF, byte >> 4), 2).reshape(last, d).long()
                sign = 1.0 - 2.0 * (nibble >> 3)
                power = torch.exp2(s["scales"][pages, which, h].reshape(-1, d // 32)[:last].double() - 127.0)
                kv.append(sign * held[nibble & 7] * power.repeat_interleave(32, 1))
            for g in range(group):
                score = s["q"][mine, (h * group + g) * d:(h * group + g + 1) * d].double() @ kv[0].T / math.sqrt(d)
                out[mine, h * group + g] = torch.softmax(score.masked_fill(~seen, -math.inf), 1) @ kv[1]
    return out.reshape(m, -1)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    e, m, d, heads = SIZE[case["dtype"]], _rows_of(case), case["dim"], case["heads"]
    tokens = m * {"rows": 4, "each": 4, "map": 4, "prompt": 8}[case["how"]] + 4 * case["streams"]
    held = d // 2 + d // 32                             # bytes of a token's keys, or values, of a head
    if case["op"] == "attend":
        pairs, wanted = _keys(case)
        return {"bytes": 2 * m * case["q_heads"] * d * e + wanted * heads * 2 * held + tokens, "flops": 4 * pairs * case["q_heads"] * d}
    turning = min(m, case["length"] if case["how"] == "map" else m) * case["rot"] * 4
    per_value = (6 if case["norm"] != "none" else 0) + (3 if case["rot"] else 0)
    if case["op"] == "heads":
        values = m * (case["q_heads"] + heads) * d
        return {"bytes": 2 * values * e + turning + tokens, "flops": max(1, values * per_value)}
    values = m * heads * d
    # keys and values read, the cache written, what it holds returned
    return {"bytes": 4 * values * e + 2 * m * heads * held + turning + tokens, "flops": values * (per_value + 2 * 6)}
