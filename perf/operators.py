"""The row operators that are measured: norms around a block, and products in 8-bit integers.

A row is the channel vector of one token: one pixel of an NHWC feature map, where a list of pixel indices with its
length on the GPU names the flagged ones, or one row of a plain matrix.  Three kinds of case:

  norm     y = x + scale * gate * post(h), z = pre(y): the end of one residual block and the start of the next
  product  y = act((q . W) * row scale * channel scale + bias) of rows that are 8-bit integers already
  linear   the same product of floating-point rows: normed (or not), quantised with a scale for each row, multiplied

Rows are quantised as q = round_half_even(v * (127 / max|v|)) with the scale max|v| / 127.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
SCALE = 0.5                                             # residual scale of the norm cases
MAX_FLOPS, MAX_ELEMENTS = 1.0e12, 16384 * 4096          # what a drawn case may cost


def listed():
    return [
        # one token of the width that ends the ResNet-50-shaped backbone: latency
        _norm("norm_one_token", rows=1, c=2048, dtype="f16", post="rms", pre="rms", gate="channel"),
        # flagged pixels of 64 streams of 64x64 at 10 % density, 256 channels, a gate for each stream
        _norm("norm_flagged_pixels", rows=0, c=256, dtype="f16", post="layer", pre="layer", gate="stream", streams=64, side=64, density=0.1),
        # an odd width, whose rows start at no multiple of 16 bytes, in fp32; a plain norm before a block
        _norm("norm_odd_width", rows=4099, c=1037, dtype="f32", post="none", pre="layer", gate="none"),
        # every token of a long batch
        _norm("norm_long_batch", rows=16384, c=4096, dtype="bf16", post="rms", pre="rms", gate="channel"),
        # one token: the weights are all there is to read
        _product("product_one_token", rows=1, k=4096, n=4096, dtype="f16", act="none"),
        # the tokens of a small serving batch
        _product("product_few_tokens", rows=24, k=2048, n=8192, dtype="bf16", act="relu"),
        # nothing a multiple of anything
        _product("product_ragged", rows=1021, k=1000, n=1531, dtype="f32", act="relu6"),
        # a long batch
        _product("product_long_batch", rows=16384, k=4096, n=4096, dtype="bf16", act="relu"),
        # one token from the residual stream: norm, 8-bit row and product
        _linear("linear_one_token", rows=1, k=4096, n=4096, dtype="bf16", act="none", norm="rms"),
        # the channel expansion of a block on the flagged pixels of 64 streams of 64x64
        _linear("linear_flagged_pixels", rows=0, k=256, n=1024, dtype="f16", act="relu", norm="layer", streams=64, side=64, density=0.1),
        # the update of a few streams, or a short prompt
        _linear("linear_short_prompt", rows=500, k=2048, n=8192, dtype="f16", act="relu", norm="rms"),
        # hidden rows of a block in a long batch: quantised between its two products
        _linear("linear_long_batch", rows=8192, k=8192, n=4096, dtype="f16", act="none", norm="none"),
    ]


def _norm(name, rows, c, dtype, post, pre, gate, streams=0, side=0, density=0.0):
    return dict(name=name, op="norm", rows=rows, c=c, dtype=dtype, post=post, pre=pre, gate=gate, streams=streams, side=side, density=density)


def _product(name, rows, k, n, dtype, act):
    return dict(name=name, op="product", rows=rows, k=k, n=n, dtype=dtype, act=act, streams=0, side=0, density=0.0)


def _linear(name, rows, k, n, dtype, act, norm, streams=0, side=0, density=0.0):
    return dict(name=name, op="linear", rows=rows, k=k, n=n, dtype=dtype, act=act, norm=norm, streams=streams, side=side, density=density)


def draw(rng):
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["norm", "product", "linear"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    on_map = op != "product" and rng.random() < 0.4
    streams, side, density = (rng.randint(1, 64), rng.randint(8, 64), rng.choice([0.03, 0.1, 0.3])) if on_map else (0, 0, 0.0)
    rows = 0 if on_map else spread(1, 16384)
    about = max(1, int(streams * side * side * density)) if on_map else rows
    if op == "norm":
        c = min(spread(32, 8192), MAX_ELEMENTS // max(about, streams * side * side))
        post, pre = rng.choice(["none", "rms", "layer"]), rng.choice(["rms", "layer"])
        return {k: v for k, v in _norm("", rows, c, dtype, post, pre, rng.choice(["none", "channel", "stream"]) if on_map else rng.choice(["none", "channel"]),
                                       streams, side, density).items() if k != "name"}
    act = rng.choice(["none", "relu", "relu6"])
    while True:
        k, n = spread(64, 8192), spread(64, 8192)
        if 2.0 * about * k * n <= MAX_FLOPS / 4 and max(about, streams * side * side) * max(k, n) <= MAX_ELEMENTS:
            break
    if op == "product":
        case = _product("", rows, k, n, dtype, act)
    else:
        # fp32 rows come without a norm: a norm's last bit moves an 8-bit value that lies between two, and with it an fp32 result
        norm = "none" if dtype == "f32" else rng.choice(["none", "rms", "layer"])
        case = _linear("", rows, k, n, dtype, act, norm, streams, side, density)
    return {k: v for k, v in case.items() if k != "name"}


def _pixels(case):
    """Pixels of a case's map, and how many of them are flagged."""
    px = case["streams"] * case["side"] ** 2
    return px, max(1, round(px * case["density"]))


def _flagged(case, gen):
    """The list of a map's flagged pixels as the library keeps one (room for all, the first `m` valid), its length and m."""
    px, m = _pixels(case)
    idx = torch.zeros(px, dtype=torch.int32, device="cuda")
    idx[:m] = torch.randperm(px, device="cuda", generator=gen)[:m].sort().values
    return idx, torch.tensor([m], dtype=torch.int32, device="cuda"), m


def _rows(case, gen, rows, c):
    """Rows of a residual stream: channels of different scales, a few of them far larger than the rest."""
    by_channel = torch.exp(0.5 * torch.randn(c, device="cuda", generator=gen))
    by_channel[torch.randperm(c, device="cuda", generator=gen)[:max(1, c // 256)]] *= 12.0
    return (torch.randn(rows, c, device="cuda", generator=gen) * by_channel).to(DTYPES[case["dtype"]])


def _about(case, gen, c, mean):
    return (mean + 0.1 * torch.randn(c, device="cuda", generator=gen)).to(DTYPES[case["dtype"]])


def _weights(gen, k, n):
    """8-bit weights [k, n] with a scale for each channel."""
    w = torch.randn(k, n, device="cuda", generator=gen)
    scale = w.abs().amax(0) / 127.0
    q = torch.round(w / scale).clamp_(-127, 127).to(torch.int8)
    return q, scale * (1.0 / math.sqrt(k))


def _norm_parameters(case, gen, kind, c):
    if kind == "none":
        return None
    return kind, _about(case, gen, c, 1.0), _about(case, gen, c, 0.0) if kind == "layer" else None


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case, "idx": None, "count": None, "m": case["rows"]}
    rows = case["rows"]
    if case["streams"]:
        s["idx"], s["count"], s["m"] = _flagged(case, gen)
        rows = case["streams"] * case["side"] ** 2
    if case["op"] == "norm":
        c = case["c"]
        s["x"] = _rows(case, gen, rows, c)
        s["h"] = _rows(case, gen, s["m"], c)
        s["post"], s["pre"] = _norm_parameters(case, gen, case["post"], c), _norm_parameters(case, gen, case["pre"], c)
        s["gate"] = {"none": lambda: None, "channel": lambda: _about(case, gen, c, 0.3),
                     "stream": lambda: (0.3 + 0.1 * torch.randn(case["streams"], c, device="cuda", generator=gen)).to(DTYPES[case["dtype"]])}[case["gate"]]()
        s["gate_rows"] = case["side"] ** 2 if case["gate"] == "stream" else 0
        s["y"] = s["x"].clone()                         # pixels that are not listed keep their rows
    else:
        k, n = case["k"], case["n"]
        s["w"], s["w_scale"] = _weights(gen, k, n)
        s["bias"] = (0.1 * torch.randn(n, device="cuda", generator=gen)).to(DTYPES[case["dtype"]])
        if case["op"] == "product":
            x = torch.randn(rows, k, device="cuda", generator=gen)
            s["scale"] = x.abs().amax(1) / 127.0
            wide = torch.zeros(rows, -(-k // 16) * 16, dtype=torch.int8, device="cuda")
            wide[:, :k] = torch.round(x / s["scale"][:, None]).clamp_(-127, 127).to(torch.int8)
            s["q"] = wide[:, :k]
        else:
            s["x"] = _rows(case, gen, rows, k)
            s["pre"] = _norm_parameters(case, gen, case["norm"], k)
    if own:
        import paper_2203_03996_amd as pkg
        s["ctx"] = ctx = pkg.Context(0)
        if case["op"] == "norm":
            s["post"], s["pre"] = (p and pkg.RowNorm(*p, eps=EPS) for p in (s["post"], s["pre"]))
        else:
            s["weights"] = pkg.RowWeights(ctx, s["w"], scale=s["w_scale"], bias=s["bias"], act=case["act"])
            if case["op"] == "linear":
                s["pre"] = s["pre"] and pkg.RowNorm(*s["pre"], eps=EPS)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _normed(v, p):
    """v in 32 bits, p = (kind, weight, bias) or None."""
    if p is None:
        return v
    kind, w, b = p
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * w.float()
    return v if b is None else v + b.float()


def _product_of(s, q, scale):
    y = torch.matmul(q, s["w"].float()) * (scale[:, None] * s["w_scale"]) + s["bias"].float()
    if s["case"]["act"] == "relu":
        y = torch.clamp(y, min=0.0)
    elif s["case"]["act"] == "relu6":
        y = torch.clamp(y, 0.0, 6.0)
    return y.to(DTYPES[s["case"]["dtype"]])


def _plain(s):
    case, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    at = None if s["idx"] is None else s["idx"][:s["m"]].long()
    if case["op"] == "product":
        return _product_of(s, s["q"].float(), s["scale"])
    x = (s["x"] if at is None else s["x"][at]).float()
    if case["op"] == "norm":
        p = _normed(s["h"].float(), s["post"])
        if s["gate"] is not None:
            p = p * (s["gate"] if not s["gate_rows"] else s["gate"][at // s["gate_rows"]]).float()
        y = x + SCALE * p
        z = _normed(y, s["pre"]).to(dtype)
        if at is None:
            s["y"] = y.to(dtype)
        else:
            s["y"][at] = y.to(dtype)
        return s["y"], z
    v = _normed(x, s["pre"])
    amax = v.abs().amax(1)
    # (a division of two tensors: `127.0 / amax` would round twice)
    q = torch.round(v * (torch.full_like(amax, 127.0) / amax)[:, None]).clamp_(-127, 127)
    return _product_of(s, q, amax / 127.0)


def run(s):
    if not own:
        return _plain(s)
    case = s["case"]
    if case["op"] == "norm":
        y, z, _, _ = s["ctx"].rows_norm(s["x"], s["h"], post=s["post"], gate=s["gate"], gate_rows=s["gate_rows"], scale=SCALE, pre=s["pre"],
                                        idx=s["idx"], count=s["count"], y=s["y"], z=True)
        return y, z[:s["m"]]
    if case["op"] == "product":
        return s["weights"].matmul(s["q"], s["scale"], dtype=DTYPES[case["dtype"]])
    return s["weights"].linear(s["x"], pre=s["pre"], idx=s["idx"], count=s["count"])[:s["m"]]


# ---- the definition in 64 bits --------------------------------------------------------------------------------------
def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    f64 = torch.float64

    def norm64(v, p):
        if p is None:
            return v
        kind, w, b = p
        c = v.shape[1]
        centred = v - v.sum(1, keepdim=True) / c if kind == "layer" else v
        spread = torch.sqrt(centred.square().sum(1, keepdim=True) / c + EPS)
        out = centred / spread * w.to(f64)
        return out + b.to(f64) if b is not None else out

    at = None if s["idx"] is None else s["idx"][:s["m"]].long()
    if case["op"] == "norm":
        x = s["x"].to(f64)
        p = norm64(s["h"].to(f64), s["post"])
        if s["gate"] is not None:
            gate = s["gate"].to(f64)
            p = p * (gate[torch.div(at, s["gate_rows"], rounding_mode="floor")] if s["gate_rows"] else gate)
        if at is None:
            y = listed_y = x + SCALE * p
        else:
            listed_y = x[at] + SCALE * p
            y = x.index_copy(0, at, listed_y)
        return y, norm64(listed_y, s["pre"])
    if case["op"] == "product":
        q, scale = s["q"].to(f64), s["scale"].to(f64)
    else:
        v = norm64((s["x"] if at is None else s["x"][at]).to(f64), s["pre"])
        scale = v.abs().amax(1) / 127.0
        q = torch.round(v / scale[:, None])
    y = (q @ s["w"].to(f64)) * scale[:, None] * s["w_scale"].to(f64) + s["bias"].to(f64)
    if case["act"] != "none":
        y = y.clamp(0.0, 6.0 if case["act"] == "relu6" else math.inf)
    return y


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    e = SIZE[case["dtype"]]
    m = _pixels(case)[1] if case["streams"] else case["rows"]
    listing = 4 * m + 4 if case["streams"] else 0
    if case["op"] == "norm":
        c = case["c"]
        vectors = sum((kind != "none") + (kind == "layer") for kind in (case["post"], case["pre"]))
        vectors += {"none": 0, "channel": 1, "stream": case["streams"]}[case["gate"]]
        # x and h read, y and z written; a norm takes about 6 operations an element, gate and residual 3
        return {"bytes": 4 * m * c * e + vectors * c * e + listing, "flops": m * c * (3 + 6 * ((case["post"] != "none") + (case["pre"] != "none")))}
    k, n = case["k"], case["n"]
    rows = m * (k + 4) if case["op"] == "product" else m * k * e + listing
    if case["op"] == "linear":
        rows += k * e * ((case["norm"] != "none") + (case["norm"] == "layer"))
    return {"bytes": rows + k * n + 4 * n + n * e + m * n * e, "flops": 2 * m * k * n}
