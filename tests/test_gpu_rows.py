"""Row operators (norms around a block, rows in 8 bits, products in 8-bit integers) against plain forms in 64 bits.

Tolerances follow from the arithmetic.  U32 and U are the unit round-offs of fp32 and of the storage type:
* norms: a lane adds at most 64 numbers in a row and ten more steps join the lanes, so a sum of magnitudes is good to
  74 U32 and a norm's factor to half of that; with the few products and sums behind it 128 U32 of the magnitudes that
  meet in an element bounds the fp32 part, and one rounding to the storage type adds U of the result.
* products: the integer sums are exact; the conversion of the sum, the product of the scales, the product of both and
  the sum with the bias are one rounding each: 4 U32 of the magnitudes that meet, and U of the result.
* results below the storage type's normal range are good to half of its smallest step."""
import numpy as np
import pytest
import torch

import paper_2203_03996_amd as pkg

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
TYPES = {"f32": (torch.float32, 2.0 ** -24, 2.0 ** -149), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -133)}
# (8 bits of significand in bf16, 11 in f16, 24 in f32: round-off half a unit of the last)


@pytest.fixture(scope="module")
def ctx():
    return pkg.Context(0)


def np64(t):
    return t.detach().double().cpu().numpy()


def rand(rng, shape, dt, scale=1.0, mean=0.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale + mean).astype(np.float32)).to(TYPES[dt][0]).cuda()


def close(got, want, dt, slack, what):
    _, u, tiny = TYPES[dt]
    got, err = np64(got), None
    assert got.shape == want.shape, what
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    with np.errstate(invalid="ignore"):
        err = np.abs(got - want) - (u * np.abs(want) + slack + 0.5 * tiny)
    assert not fine.any() or err[fine].max() <= 0, f"{what}: off by {err[fine].max():.3e} more than the arithmetic allows (at {np.argwhere(err == err[fine].max())[0]})"


def norm64(v, kind, w, b, eps):
    """(norm of the rows of v, magnitudes that meet in its elements)"""
    if kind == "none":
        return v, np.abs(v)
    top = np.abs(v).max(1, keepdims=True, initial=0.0)
    d = v - v.mean(1, keepdims=True) if kind == "layer" else v
    f = 1.0 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    w = np.ones(v.shape[1]) if w is None else w
    b = np.zeros(v.shape[1]) if b is None else b
    return d * f * w + b, top * f * np.abs(w) + np.abs(b)


def factor64(v, kind, w, eps):
    """What an error of an element of v becomes in its norm, at most (the row's common factor; the statistics follow the same bound)."""
    if kind == "none":
        return np.ones_like(v)
    d = v - v.mean(1, keepdims=True) if kind == "layer" else v
    return 2.0 / np.sqrt((d * d).mean(1, keepdims=True) + eps) * (np.ones(v.shape[1]) if w is None else np.abs(w))


class NormCase:
    """Inputs of rows_norm, and what 64 bits make of them."""

    def __init__(self, dt, rows, c, post="rms", pre="rms", gate="channel", params=True, on_map=False, seed=0, mean=0.0, eps=1e-5, scale=0.75):
        rng = np.random.default_rng([seed, rows, c])
        self.dt, self.c, self.eps, self.scale = dt, c, eps, scale
        self.map_rows = 3 * rows + 5 if on_map else rows
        self.idx = self.count = None
        self.at = np.arange(rows)
        if on_map:
            self.at = np.sort(rng.choice(self.map_rows, rows, replace=False))
            room = np.full(rows + 7, 1 << 30, np.int32)              # entries behind the list's end name nothing
            room[:rows] = self.at
            self.idx = torch.from_numpy(room).cuda()
            self.count = torch.tensor([rows], dtype=torch.int32, device="cuda")
        self.x = rand(rng, (self.map_rows, c), dt, 2.0, mean)
        self.h = rand(rng, (rows, c), dt, 3.0, mean)
        self.gate_rows = {"none": 0, "channel": 0, "group": 4, "row": 1}[gate]
        groups = -(-self.map_rows // self.gate_rows) if self.gate_rows else 1
        self.gate = None if gate == "none" else rand(rng, (groups, c), dt, 0.5)
        self.norms, self.p64 = [], []
        for kind in (post, pre):
            w = rand(rng, c, dt, 0.3, 1.0) if params else None
            b = rand(rng, c, dt, 0.3) if params and kind == "layer" else None
            self.norms.append(pkg.RowNorm(kind, w, b, eps) if kind != "none" else None)
            self.p64.append((kind, None if w is None else np64(w), None if b is None else np64(b), eps))

    def want(self):
        x, h = np64(self.x)[self.at], np64(self.h)
        p, mag = norm64(h, *self.p64[0])
        g = np.ones_like(p) if self.gate is None else np64(self.gate)[self.at // self.gate_rows if self.gate_rows else np.zeros_like(self.at)]
        y = x + self.scale * g * p
        y_slack = 128 * U32 * (np.abs(x) + np.abs(self.scale * g) * mag)
        z, zmag = norm64(y, *self.p64[1])
        z_slack = 128 * U32 * zmag + y_slack.max(1, keepdims=True) * factor64(y, self.p64[1][0], self.p64[1][1], self.eps)
        return y, y_slack, z, z_slack

    def run(self, ctx, **kw):
        return ctx.rows_norm(self.x, self.h, post=self.norms[0], gate=self.gate, gate_rows=self.gate_rows, scale=self.scale, pre=self.norms[1],
                             idx=self.idx, count=self.count, **kw)

    def check(self, ctx, what=""):
        y0 = torch.full_like(self.x, 7.0)
        rows = len(self.at)
        y, z, q, qs = self.run(ctx, y=y0, z=True, q=True)
        ctx.sync()
        y64, ys, z64, zs = self.want()
        close(y[torch.from_numpy(self.at).cuda()], y64, self.dt, ys, f"{what} y")
        rest = np.ones(self.map_rows, bool)
        rest[self.at] = False
        assert (np64(y)[rest] == 7.0).all(), f"{what}: a row that is not listed was written"
        close(z[:rows], z64, self.dt, zs, f"{what} z")
        check_q(q[:rows], qs[:rows], z64, zs, f"{what} q")


def check_q(q, qs, z64, zs, what):
    """8-bit rows against the values that they stand for: half a step off, plus what the values themselves may be off."""
    q, qs = np64(q), np64(qs)[:, None]
    amax = np.abs(z64).max(1, keepdims=True)
    assert (np.abs(qs - amax / 127) <= zs.max(1, keepdims=True) / 127 + 4 * U32 * amax / 127).all(), f"{what}: scale"
    assert (np.abs(q * qs - z64) <= qs * (0.5 + 127 * 4 * U32) + 2 * zs.max(1, keepdims=True)).all(), f"{what}: values"
    assert (np.abs(q).max(1) == 127).all(), f"{what}: the largest magnitude of a row is 127"


WIDTHS = [1, 2, 7, 8, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 300, 511, 512, 513, 1000, 1024, 1037, 2048, 2049, 4095, 4096, 5000, 8192, 8193, 16384,
          16391, 32768]


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("c", WIDTHS)
def test_norm_widths(ctx, dt, c):
    NormCase(dt, 5, c, "layer", "rms", "channel").check(ctx, f"{dt} c={c}")
    if c > 1:                                                       # (a layer norm over one channel is 0 everywhere: nothing to scale by)
        NormCase(dt, 3, c, "rms", "layer", "row", on_map=True).check(ctx, f"{dt} c={c} map")


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 31, 33, 64, 100, 257, 3001])
def test_norm_rows(ctx, dt, rows):
    NormCase(dt, rows, 64, "rms", "layer", "group", on_map=True).check(ctx, f"rows={rows} c=64")
    NormCase(dt, rows, 200, "layer", "rms", "channel").check(ctx, f"rows={rows} c=200")
    NormCase(dt, min(rows, 257), 2100, "none", "layer", "none").check(ctx, f"rows={rows} c=2100")


@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("gate", ["none", "channel", "group", "row"])
def test_norm_forms(ctx, post, pre, gate):
    NormCase("f16", 37, 96, post, pre, gate, on_map=True).check(ctx, f"{post} {pre} {gate}")
    NormCase("f32", 11, 1500, post, pre, gate, params=False).check(ctx, f"{post} {pre} {gate} no parameters")


@pytest.mark.parametrize("dt", list(TYPES))
def test_norm_offset_rows_keep_their_variance(ctx, dt):
    """Rows far from zero: the variance comes from centred values, not from a difference of squares."""
    NormCase(dt, 9, 384, "layer", "layer", "channel", mean=100.0).check(ctx, f"{dt} mean 100")


def test_norm_of_rows_without_a_block(ctx):
    """h is None: z and q of x alone; and y of a block without a residual."""
    case = NormCase("bf16", 21, 80, on_map=True)
    _, z, q, qs = ctx.rows_norm(case.x, pre=case.norms[1], idx=case.idx, count=case.count, z=True, q=True)
    ctx.sync()
    x = np64(case.x)[case.at]
    want, mag = norm64(x, *case.p64[1])
    close(z[:21], want, "bf16", 128 * U32 * mag, "z")
    check_q(q[:21], qs[:21], want, 128 * U32 * mag, "q")
    y, _, _, _ = ctx.rows_norm(None, case.h, post=case.norms[0], scale=0.5, y=True)
    ctx.sync()
    want, mag = norm64(np64(case.h), *case.p64[0])
    close(y, 0.5 * want, "bf16", 128 * U32 * mag, "y")


def test_norm_in_place_and_strided(ctx):
    """y is x itself; every matrix is a view with a leading dimension of its own that starts at an odd element."""
    for dt in TYPES:
        case = NormCase(dt, 19, 133, "rms", "layer", "group", on_map=True)
        y64, ys, z64, zs = case.want()

        def view(t, pad):
            wide = torch.full((t.shape[0], t.shape[1] + pad + 1), 5.0, dtype=t.dtype, device="cuda")
            wide[:, 1:1 + t.shape[1]] = t
            return wide, wide[:, 1:1 + t.shape[1]]
        xw, case.x = view(case.x, 4)
        _, case.h = view(case.h, 2)
        _, case.gate = view(case.gate, 6)
        zw, z = view(torch.zeros(26, 133, dtype=case.h.dtype, device="cuda"), 9)
        before = np64(case.x)
        case.run(ctx, y=case.x, z=z)
        ctx.sync()
        close(case.x[torch.from_numpy(case.at).cuda()], y64, dt, ys, "y")
        close(z[:19], z64, dt, zs, "z")
        rest = np.ones(case.map_rows, bool)
        rest[case.at] = False
        assert np.array_equal(np64(case.x)[rest], before[rest])
        for w in (xw, zw):
            assert (np64(w)[:, 0] == 5.0).all() and (np64(w)[:, 134:] == 5.0).all(), "columns beside the rows were written"
        assert (np64(z)[19:] == 0.0).all(), "rows behind the count were written"


@pytest.mark.parametrize("dt,widths", [("f16", (513, 1025, 1029, 2049, 4097, 8195)), ("bf16", (1025, 4100)), ("f32", (257, 513, 514, 1025, 4097))])
def test_norm_in_place_at_odd_widths(ctx, dt, widths):
    """A row's last vector shares elements with the one before it, which another wave may hold: nothing is written that is still to be read."""
    for c in widths:
        for post in ("none", "rms"):
            case = NormCase(dt, 300, c, post, "rms", "none", seed=4)
            y64, ys, z64, zs = case.want()
            case.run(ctx, y=case.x, z=True)
            ctx.sync()
            close(case.x, y64, dt, ys, f"c={c} post {post}")


def test_norm_lists(ctx):
    """Counts of zero, below zero and beyond the room; entries that name no row."""
    case = NormCase("f16", 40, 72, on_map=True)
    y64, ys, z64, zs = case.want()
    for count, n in ((0, 0), (-3, 0), (17, 17), (40, 40)):
        case.count.fill_(count)
        y, z, q, qs = case.run(ctx, y=torch.full_like(case.x, 7.0), z=torch.full((47, 72), 9.0, dtype=torch.float16, device="cuda"), q=True)
        ctx.sync()
        listed = case.at[:n]
        rest = np.ones(case.map_rows, bool)
        rest[listed] = False
        assert (np64(y)[rest] == 7.0).all() and (np64(z)[n:] == 9.0).all()
        close(z[:n], z64[:n], "f16", zs[:n], f"count {count}")
        close(y[torch.from_numpy(listed).cuda()], y64[:n], "f16", ys[:n], f"count {count}")
    case.count.fill_(1 << 20)                                      # more than there is room for: h has 40 rows
    drop = np.array([0, 5, 39])
    case.idx[torch.from_numpy(drop).cuda()] = torch.tensor([-1, case.map_rows, -(1 << 31)], dtype=torch.int32, device="cuda")
    y, z, q, qs = case.run(ctx, y=torch.full_like(case.x, 7.0), z=True, q=True)
    ctx.sync()
    keep = np.setdiff1d(np.arange(40), drop)
    assert z.shape[0] == 40
    assert (np64(z)[drop] == 0).all() and (np64(q)[drop] == 0).all() and (np64(qs)[drop] == 0).all()
    close(z[torch.from_numpy(keep).cuda()], z64[keep], "f16", zs[keep], "kept rows")
    rest = np.ones(case.map_rows, bool)
    rest[case.at[keep]] = False
    assert (np64(y)[rest] == 7.0).all()


def plain_q(x):
    """The definition, step by step in fp32 (numpy's division and product are rounded once each, as the kernels' are)."""
    x = x.astype(np.float32)
    amax = np.abs(x).max(1, keepdims=True)
    return np.rint(x * (np.float32(127.0) / amax)).astype(np.int64), amax[:, 0].astype(np.float64) / 127


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("c", [1, 8, 33, 64, 500, 2048, 6001])
def test_quantize_is_the_definition_bit_for_bit(ctx, dt, c):
    rng = np.random.default_rng(c)
    x = rand(rng, (77, c), dt, 4.0)
    x[:, 0] = x[:, 0] * 8
    x[np.abs(np64(x)).max(1) == 0] = 1.0
    q, qs = ctx.rows_quantize(x)
    ctx.sync()
    want, scale = plain_q(x.float().cpu().numpy())
    assert np.array_equal(np64(q), want)
    assert np.abs(np64(qs) - scale).max() <= U32 * scale.max() and (np.abs(np64(qs) / scale - 1) <= 2 * U32).all()


def test_quantize_ties_go_to_even(ctx):
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5, -126.5, 3.49999, 3.50001]], device="cuda")
    q, qs = ctx.rows_quantize(x)
    ctx.sync()
    assert np64(q).tolist() == [[127, 0, 2, 2, 0, -2, -2, 126, -126, 3, 4]] and float(qs[0]) == 1.0


def test_quantize_of_empty_tiny_huge_and_broken_rows(ctx):
    """Rows of zeros, below and above the smallest scale, of the largest numbers, with infinities and NaN."""
    big = float(np.finfo(np.float32).max)
    x = torch.zeros(9, 40, device="cuda")
    x[1, 3] = 9e-37
    x[2, 3], x[2, 4] = 2e-36, -1e-36
    x[3, 0], x[3, 1] = big, -big
    x[4, 39] = float("inf")
    x[5, 39] = float("-inf")
    x[6, 0] = float("nan")
    x[7, 0], x[7, 39] = float("nan"), float("inf")
    x[8, 5] = -1.0
    q, qs = ctx.rows_quantize(x)
    ctx.sync()
    q, qs = np64(q), np64(qs)
    assert (q[[0, 1, 4, 5, 6, 7]] == 0).all()
    assert (qs[[0, 1]] == 0).all() and np.isnan(qs[4:8]).all()
    assert q[2, 3] == 127 and q[2, 4] in (-63, -64) and q[3, 0] == 127 and q[3, 1] == -127 and np.isfinite(qs[3])
    assert q[8].tolist() == [0] * 5 + [-127] + [0] * 34


def test_norm_of_broken_rows_stays_in_the_row(ctx):
    """A NaN or an infinity reaches its own row only."""
    case = NormCase("f32", 6, 90, "rms", "layer")
    case.h[1, 7] = float("nan")
    case.x[3, 8] = float("inf")
    y, z, q, qs = case.run(ctx, y=True, z=True, q=True)
    ctx.sync()
    good = [0, 2, 4, 5]
    y64, ys, z64, zs = case.want()
    close(z[good], z64[good], "f32", zs[good], "z")
    assert np.isnan(np64(z)[[1, 3]]).all() and np.isnan(np64(y)[1]).all() and np.isinf(np64(y)[3, 8])
    assert np.isnan(np64(qs)[[1, 3]]).all() and (np64(q)[[1, 3]] == 0).all()


# ---- products -------------------------------------------------------------------------------------------------------
def q_rows(rng, rows, k):
    """8-bit rows in storage whose bytes behind k hold anything, and their scales."""
    wide = torch.from_numpy(rng.integers(-127, 128, (rows, -(-k // 16) * 16), dtype=np.int8)).cuda()
    return wide[:, :k], torch.from_numpy(rng.uniform(0.5, 2.0, rows).astype(np.float32)).cuda()


def q_weights(rng, k, n):
    return (torch.from_numpy(rng.integers(-127, 128, (k, n), dtype=np.int8)).cuda(),
            torch.from_numpy((rng.uniform(0.5, 2.0, n) / (5000 * np.sqrt(k))).astype(np.float32)).cuda())


def act64(v, act):
    return v if act == "none" else np.clip(v, 0.0, 6.0 if act == "relu6" else None)


def product64(q, qs, w, ws, bias, act):
    s = np64(q) @ np64(w) * np64(qs)[:, None] * np64(ws)
    b = np.zeros(w.shape[1]) if bias is None else np64(bias)
    return act64(s + b, act), 4 * U32 * (np.abs(s) + np.abs(b))


def check_product(ctx, rng, dt, rows, k, n, act="none", with_bias=True):
    q, qs = q_rows(rng, rows, k)
    w, ws = q_weights(rng, k, n)
    bias = rand(rng, n, dt, 0.5) if with_bias else None
    weights = pkg.RowWeights(ctx, w, scale=ws, bias=bias, act=act)
    y = weights.matmul(q, qs, dtype=TYPES[dt][0])
    ctx.sync()
    want, slack = product64(q, qs, w, ws, bias, act)
    close(y, want, dt, slack, f"{dt} {rows}x{k}x{n} {act}")


ROWS = [1, 2, 3, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 200, 256, 257, 300]
KS = [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 300, 1000, 1024, 2047]
NS = [1, 2, 3, 5, 31, 32, 33, 64, 65, 100, 127, 128, 129, 256, 257, 500]


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows", ROWS)
def test_product_rows(ctx, dt, rows):
    rng = np.random.default_rng(rows)
    check_product(ctx, rng, dt, rows, 300, 100, "relu")
    check_product(ctx, rng, dt, rows, 1024, 257, "none")


@pytest.mark.parametrize("rows", [1, 7, 40, 150])
@pytest.mark.parametrize("k", KS)
def test_product_k(ctx, rows, k):
    check_product(ctx, np.random.default_rng(k), "f32", rows, k, 70, "none", with_bias=False)


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("n", NS)
def test_product_n(ctx, dt, n):
    rng = np.random.default_rng(n)
    for rows in (1, 20, 130):
        check_product(ctx, rng, dt, rows, 200, n, "relu6")


@pytest.mark.parametrize("rows,k,n", [(1, 16384, 64), (1, 65536, 33), (4, 8192, 4096), (16, 12000, 96), (24, 2048, 8192), (60, 4096, 1000), (500, 2048, 3000),
                                      (1021, 1000, 1531), (2000, 512, 2049), (3000, 256, 700), (5, 64, 70000), (2500, 4100, 2300)])
def test_product_large(ctx, rows, k, n):
    """Shapes on every side of the rules that pick a kernel."""
    check_product(ctx, np.random.default_rng(rows), "f32", rows, k, n, "relu")
    check_product(ctx, np.random.default_rng(rows), "bf16", rows, k, n, "none")


@pytest.mark.parametrize("rows,k,n", [(2000, 1200, 1500), (4100, 700, 4100), (4100, 1100, 4400), (9000, 300, 4100), (8200, 1100, 8200), (2300, 2500, 2100), (130, 9000, 130), (33, 16500, 70)])
def test_product_tiles(ctx, rows, k, n):
    """Every size of tile, workgroups with several of them, even and odd numbers of K-tiles; all rows, a part of them by a count on the GPU.
    (The reference in 64 bits is of some rows, on the GPU: a product of whole numbers below 2^53.)"""
    rng = np.random.default_rng(rows)
    q, qs = q_rows(rng, rows, k)
    w, ws = q_weights(rng, k, n)
    bias = rand(rng, n, "f32")
    weights = pkg.RowWeights(ctx, w, scale=ws, bias=bias)
    for count in (rows, max(1, rows - 37), min(70, rows), 1):
        out = torch.full((rows, n), 3.0, device="cuda")
        weights.matmul(q, qs, out=out, dtype=torch.float32, count=torch.tensor([count], dtype=torch.int32, device="cuda") if count < rows else None)
        ctx.sync()
        some = np.unique(np.concatenate([np.arange(min(count, 40)), rng.integers(0, count, 200), np.arange(max(0, count - 40), count)]))
        at = torch.from_numpy(some).cuda()
        s = (q[at].double() @ w.double()) * qs[at].double()[:, None] * ws.double()
        close(out[at], np64(s + bias.double()), "f32", np64(4 * U32 * (s.abs() + bias.double().abs())), f"{rows}x{k}x{n} count {count}")
        assert (out[count:] == 3.0).all()


def test_product_sums_are_exact_at_their_largest(ctx):
    """Every product at its largest magnitude over the longest k: 65536 * 127 * 127 and 65536 * 128 * 128 fit 32 bits."""
    for rows in (1, 3, 20, 140):
        for a, b in ((127, 127), (-128, -128), (-128, 127)):
            q = torch.full((rows, 65536), a, dtype=torch.int8, device="cuda")
            w = torch.full((65536, 40), b, dtype=torch.int8, device="cuda")
            one = torch.ones(65536, device="cuda")
            y = pkg.RowWeights(ctx, w, scale=one[:40]).matmul(q, one[:rows], dtype=torch.float32)
            ctx.sync()
            assert (np64(y) == np.float64(np.float32(65536 * a * b))).all()


@pytest.mark.parametrize("rows,room", [(9, 30), (40, 200), (150, 1000)])
def test_product_count_and_strides(ctx, rows, room):
    """The number of rows on the GPU, outputs in a wider matrix: what is behind the count and beside the columns stays."""
    rng = np.random.default_rng(room)
    k, n = 130, 75
    q, qs = q_rows(rng, room, k)
    w, ws = q_weights(rng, k, n)
    weights = pkg.RowWeights(ctx, w, scale=ws)
    want, slack = product64(q, qs, w, ws, None, "none")
    for count in (0, -1, 1, rows, room, room + 99):
        wide = torch.full((room, n + 6), 3.0, dtype=torch.float16, device="cuda")
        c = torch.tensor([count], dtype=torch.int32, device="cuda")
        weights.matmul(q, qs, count=c, out=wide[:, 1:1 + n])
        ctx.sync()
        m = max(0, min(count, room))
        close(wide[:m, 1:1 + n], want[:m], "f16", slack[:m], f"count {count}")
        assert (np64(wide)[m:] == 3.0).all() and (np64(wide)[:, 0] == 3.0).all() and (np64(wide)[:, 1 + n:] == 3.0).all()


@pytest.mark.parametrize("dt", list(TYPES))
def test_pack_quantises_each_channel(ctx, dt):
    """Floating-point weights: the 8-bit values of the definition, read back through products with unit rows."""
    rng = np.random.default_rng(3)
    k, n = 150, 45
    w = rand(rng, (k, n + 3), dt, 0.2)[:, 1:1 + n]                 # a view: rows lie n + 3 apart
    w[:, 7] = 0.0
    weights = pkg.RowWeights(ctx, w)
    eye = torch.zeros(k, 160, dtype=torch.int8, device="cuda")
    eye[:, :k] = torch.eye(k, dtype=torch.int8)
    y = weights.matmul(eye[:, :k], torch.ones(k, device="cuda"), dtype=torch.float32)
    ctx.sync()
    cols = [j for j in range(n) if j != 7]
    q, scale = plain_q(w.float().cpu().numpy().T[cols])
    got = np64(y)
    assert (got[:, 7] == 0).all()
    assert np.abs(got[:, cols] - q.T * scale).max() <= 4 * U32 * np.abs(got).max()


@pytest.mark.parametrize("rows", [3, 50, 300])
def test_product_of_broken_rows(ctx, rows):
    """A row whose scale is NaN gives NaN, with every activation, and no other row does."""
    rng = np.random.default_rng(rows)
    q, qs = q_rows(rng, rows, 96)
    w, ws = q_weights(rng, 96, 50)
    qs[1] = float("nan")
    q[2] = 0
    for act in ("none", "relu", "relu6"):
        bias = rand(rng, 50, "f16")
        y = pkg.RowWeights(ctx, w, scale=ws, bias=bias, act=act).matmul(q, qs)
        ctx.sync()
        assert np.isnan(np64(y)[1]).all() and not np.isnan(np64(y)[[0] + list(range(2, rows))]).any()
        assert np.array_equal(np64(y)[2], act64(np64(bias), act))


# ---- norm, 8-bit rows and product in one call -------------------------------------------------------------------------
def linear64(v, w, ws, bias, act):
    """Of rows that are quantised as the definition says, in 64 bits; and which of the 8-bit values lie so near a tie that fp32 may decide otherwise."""
    amax = np.abs(v).max(1, keepdims=True)
    at = np.divide(v * 127.0, amax, out=np.zeros_like(v), where=amax > 0)
    return act64(np.rint(at) @ np64(w) * (amax / 127) * np64(ws) + (0 if bias is None else np64(bias)), act), at, amax / 127


def check_linear(ctx, dt, rows, k, n, kind, on_map):
    rng = np.random.default_rng([rows, k])
    case = NormCase(dt, rows, k, pre=kind, on_map=on_map, seed=2)
    if on_map and rows <= 4:                                       # a list without room to spare: rows are normed on the spot
        case.idx = case.idx[:rows]
    w, ws = q_weights(rng, k, n)
    bias = rand(rng, n, dt)
    y = pkg.RowWeights(ctx, w, scale=ws, bias=bias, act="relu").linear(case.x, pre=case.norms[1], idx=case.idx, count=case.count)
    ctx.sync()
    v, mag = norm64(np64(case.x)[case.at], *case.p64[1])
    want, at, scale = linear64(v, w, ws, bias, "relu")
    # an 8-bit value within `near` of a tie may go either way: one step times its weights
    near = 127 * (128 * U32 * mag / np.maximum(np.abs(v).max(1, keepdims=True), 1e-300) + 8 * U32)
    ties = (np.abs(np.abs(at - np.floor(at)) - 0.5) <= near).astype(np.float64)
    slack = (ties @ np.abs(np64(w))) * scale * np64(ws)
    # ... and the scale of a row is as good as its largest value
    slack += (128 * U32 * mag.max(1, keepdims=True) / 127 + 8 * U32 * scale) * (np.abs(np.rint(at)) @ np.abs(np64(w))) * np64(ws) + 4 * U32 * np.abs(np64(bias))
    close(y[:rows], want, dt, slack, f"{dt} {rows}x{k}x{n} {kind}")
    if kind != "none":
        return
    # without a norm, whose sums may be formed in another order, the same bits as its two steps called one after the other
    q, qs = ctx.rows_quantize(case.x, pre=case.norms[1], idx=case.idx, count=case.count)
    two = pkg.RowWeights(ctx, w, scale=ws, bias=bias, act="relu").matmul(q, qs, dtype=TYPES[dt][0], count=case.count)
    ctx.sync()
    assert torch.equal(y[:rows], two[:rows])


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows,k,n", [(1, 64, 40), (1, 4096, 300), (2, 2048, 513), (4, 1000, 77), (7, 513, 1000), (16, 4096, 96), (17, 96, 33), (40, 300, 200), (200, 256, 1024), (700, 130, 260)])
@pytest.mark.parametrize("kind", ["none", "rms", "layer"])
@pytest.mark.parametrize("on_map", [False, True])
def test_linear(ctx, dt, rows, k, n, kind, on_map):
    check_linear(ctx, dt, rows, k, n, kind, on_map)


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("k", [1, 2, 3, 5, 7, 8, 9, 16, 17, 31, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257])
def test_linear_of_short_rows(ctx, dt, k):
    """Rows of a few channels, which one kernel norms, quantises and multiplies; on both sides of a tile of 64 tokens."""
    for rows, n, kind, on_map in ((5, 70, "rms", False), (64, 33, "none", True), (65, 200, "layer" if k > 1 else "rms", True), (150, 129, "none", False)):
        check_linear(ctx, dt, rows, k, n, kind, on_map)


@pytest.mark.parametrize("rows", [1, 6, 90])
def test_linear_of_rows_without_a_token_and_broken_rows(ctx, rows):
    rng = np.random.default_rng(rows)
    x = rand(rng, (rows + 2, 72), "f32")
    x[rows, 3] = float("nan")
    x[rows + 1] = 0.0
    idx = torch.arange(rows + 4, dtype=torch.int32, device="cuda")     # the last two name no row of x
    idx[0] = -5
    w, ws = q_weights(rng, 72, 90)
    bias = rand(rng, 90, "f32")
    weights = pkg.RowWeights(ctx, w, scale=ws, bias=bias)
    y = weights.linear(x, idx=idx)
    few = torch.cat([weights.linear(x, idx=idx[i:i + 3].contiguous()) for i in range(0, rows + 4, 3)])    # by threes: normed on the spot
    ctx.sync()
    assert np.array_equal(np64(few), np64(y), equal_nan=True)
    y = np64(y)
    assert (y[[0, rows + 1, rows + 2, rows + 3]] == np64(bias)).all() and np.isnan(y[rows]).all() and not np.isnan(y[:rows]).any()


# ---- long offsets, streams, graphs ------------------------------------------------------------------------------------
def test_offsets_beyond_32_bits(ctx):
    """Maps and compact matrices of more than 2^31 elements: rows at both ends."""
    rng = np.random.default_rng(1)
    c, rows = 8192, 270000                                         # 2.2e9 elements
    x = torch.empty(rows, c, dtype=torch.float16, device="cuda")
    at = np.array([0, 1, rows - 2, rows - 1])
    x[torch.from_numpy(at).cuda()] = rand(rng, (4, c), "f16")
    idx = torch.from_numpy(at.astype(np.int32)).cuda()
    h = rand(rng, (4, c), "f16")
    x64 = np64(x[torch.from_numpy(at).cuda()])
    w, ws = q_weights(rng, c, 40)
    y = pkg.RowWeights(ctx, w, scale=ws).linear(x, idx=idx)
    want, at_, scale = linear64(x64, w, ws, None, "none")
    ctx.rows_norm(x, h, scale=2.0, idx=idx, y=x)
    ctx.sync()
    got = x[torch.from_numpy(at).cuda()]
    close(got, x64 + 2.0 * np64(h), "f16", 128 * U32 * (np.abs(x64) + 2 * np.abs(np64(h))), "y")
    near = (np.abs(np.abs(at_ - np.floor(at_)) - 0.5) <= 127 * 16 * U32) @ np.abs(np64(w))
    close(y, want, "f16", (near + 16 * U32 * (np.abs(np.rint(at_)) @ np.abs(np64(w)))) * scale * np64(ws), "product")
    del x
    q = torch.zeros(rows, c, dtype=torch.int8, device="cuda")      # 8-bit rows of 2.2e9 bytes, outputs of 2.2e9 elements
    qs = torch.ones(rows, device="cuda")
    q[torch.from_numpy(at).cuda()] = torch.from_numpy(rng.integers(-127, 128, (4, c), dtype=np.int8)).cuda()
    wide = torch.zeros(rows, c, dtype=torch.float16, device="cuda")
    pkg.RowWeights(ctx, w, scale=ws).matmul(q, qs, out=wide[:, 11:51])
    ctx.sync()
    a = torch.from_numpy(at).cuda()
    want, slack = product64(q[a], qs[a], w, ws, None, "none")
    close(wide[a][:, 11:51], want, "f16", slack, "long product")
    assert not wide[2:rows - 2].any() and not wide[:, :11].any()


def _chain(ctx, weights, norm, x, h, out):
    ctx.rows_norm(x, h, post=norm, scale=0.5, y=out["y"], z=out["z"], q=out["q"], q_scale=out["qs"])
    weights.matmul(out["q"], out["qs"], out=out["p"])
    weights.linear(out["y"], pre=norm, out=out["l"])


@pytest.mark.parametrize("rows", [1, 12, 200])
def test_graph_replays_and_side_stream(rows):
    """A context on a stream of its own; a captured chain replayed on new inputs, with eager work in between."""
    rng = np.random.default_rng(rows)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = pkg.Context(0)
    k, n = 256, 320
    x, h = rand(rng, (rows, k), "f16"), rand(rng, (rows, k), "f16")
    w, ws = q_weights(rng, k, n)
    norm = pkg.RowNorm("rms", rand(rng, k, "f16", 0.1, 1.0))

    def buffers():
        return {"y": torch.zeros_like(x), "z": torch.zeros_like(x), "q": torch.zeros(rows, k, dtype=torch.int8, device="cuda"), "qs": torch.zeros(rows, device="cuda"),
                "p": torch.zeros(rows, n, dtype=torch.float16, device="cuda"), "l": torch.zeros(rows, n, dtype=torch.float16, device="cuda")}
    got, eager = buffers(), buffers()
    torch.cuda.synchronize()
    weights = pkg.RowWeights(ctx, w, scale=ws)                      # called while torch is on another stream
    _chain(ctx, weights, norm, x, h, got)
    ctx.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        _chain(ctx, weights, norm, x, h, got)
    for step in range(4):
        x.copy_(rand(rng, (rows, k), "f16"))
        h.copy_(rand(rng, (rows, k), "f16"))
        for t in got.values():
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        _chain(ctx, weights, norm, x, h, eager)
        ctx.sync()
        for name in got:
            assert torch.equal(got[name], eager[name]), (step, name)


@pytest.mark.parametrize("before", [None, 160])
def test_graphs_keep_their_scratch(before):
    """Captured without a call before it, or behind a small one; then larger calls without the graph, whose scratch takes the place of the first."""
    rng = np.random.default_rng(23)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = pkg.Context(0)
    k, n, rows = 4096, 128, 160                                     # (few tiles and a long k: partial sums and counts in the scratch)
    w, ws = q_weights(rng, k, n)
    x = rand(rng, (5000, k), "f16")
    torch.cuda.synchronize()
    weights = pkg.RowWeights(ctx, w, scale=ws)
    want = pkg.RowWeights(ctx, w, scale=ws).linear(x)
    if before is not None:
        weights.linear(x[:before])
    out = torch.zeros(rows, n, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        weights.linear(x[:rows], out=out)
    for eager in (rows, 200, 5000, 100):
        got = weights.linear(x[:eager])
        with torch.cuda.stream(stream):
            other = torch.full((1 << 22,), 77, dtype=torch.uint8, device="cuda")         # (in the place of scratch that was let go, if any was)
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want[:eager]) and torch.equal(out, want[:rows]) and bool((other == 77).all()), eager
        out.zero_()
        torch.cuda.synchronize()


def test_results_do_not_change_from_run_to_run(ctx):
    rng = np.random.default_rng(5)
    for rows, k, n in ((1, 8192, 512), (20, 4096, 256), (300, 1000, 500)):
        x = rand(rng, (rows, k), "bf16")
        w, ws = q_weights(rng, k, n)
        weights = pkg.RowWeights(ctx, w, scale=ws)
        first = weights.linear(x, pre=pkg.RowNorm("layer"))
        for _ in range(5):
            assert torch.equal(first, weights.linear(x, pre=pkg.RowNorm("layer")))


@pytest.mark.parametrize("order", [(3000, 100), (100, 3000, 200), (5, 20000, 64, 1, 400)])
def test_sizes_in_any_order(ctx, order):
    """Weights are called with many rows and then with few, whose k is shared out among workgroups (and their scratch is the larger one)."""
    rng = np.random.default_rng(3)
    k, n = 4096, 128
    w, ws = q_weights(rng, k, n)
    weights, other = pkg.RowWeights(ctx, w, scale=ws), pkg.RowWeights(ctx, w, scale=ws)
    x = torch.randn(max(order), k, device="cuda", dtype=torch.float16)
    q, q_scale = ctx.rows_quantize(x)
    sums = (q[:64].cpu().double() @ w.cpu().double()).numpy()
    want = sums * (np64(q_scale[:64])[:, None] * np64(ws))
    for r in order:
        for y in (weights.matmul(q[:r], q_scale[:r], dtype=torch.float32), other.linear(x[:r])):
            tol = 2.0 ** -21 if y.dtype == torch.float32 else 2.0 ** -10      # (three roundings to 24 bits; one to 11 on top of them)
            m = min(r, 64)
            assert np.abs(np64(y[:m]) - want[:m]).max() <= tol * np.abs(want).max(), (r, y.dtype)


@pytest.mark.parametrize("act", ["none", "relu6"])
@pytest.mark.parametrize("dt", list(TYPES))
def test_an_output_has_the_same_bits_whichever_kernel_makes_it(ctx, dt, act):
    """The sums are exact: how many rows there are, and so which tile or split they get, shows in nothing."""
    rng = np.random.default_rng(17)
    k, n, rows = 2048, 512, 32000
    q, qs = q_rows(rng, rows, k)
    w, ws = q_weights(rng, k, n)
    bias = rand(rng, n, dt)
    weights = pkg.RowWeights(ctx, w, scale=ws, bias=bias, act=act)
    all_rows = weights.matmul(q, qs, dtype=TYPES[dt][0])
    for r in (20000, 8000, 3000, 200, 24, 5):
        assert torch.equal(weights.matmul(q[:r], qs[:r], dtype=TYPES[dt][0]), all_rows[:r]), r


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("k", [5, 64, 77, 128, 200, 256])
def test_short_rows_have_the_same_bits_among_few_and_many(ctx, k, dt, kind):
    """Rows that a product's kernel norms for itself against rows that the norm's kernel handed over."""
    rng = np.random.default_rng(k)
    x = rand(rng, (20000, k), dt, 1.5, 0.5)
    weights = pkg.RowWeights(ctx, rand(rng, (k, 1024), "f32"))
    for norm in (pkg.RowNorm(kind), pkg.RowNorm(kind, rand(rng, k, dt), rand(rng, k, dt)), pkg.RowNorm(kind, rand(rng, k, dt))):
        all_rows = weights.linear(x, pre=norm)
        for r in (3000, 500, 40):
            assert torch.equal(weights.linear(x[:r], pre=norm), all_rows[:r]), r


@pytest.mark.parametrize("rows,n", [(8192, 1024), (2000, 300)])
def test_listed_rows_have_the_bits_of_the_whole_map(ctx, rows, n):
    """A list has room for the whole map: its length, which is on the GPU, may weigh in which kernel is taken and in nothing else."""
    rng = np.random.default_rng(rows)
    x = rand(rng, (rows, 256), "f16", 1.5, 0.5)
    weights, norm = pkg.RowWeights(ctx, rand(rng, (256, n), "f16")), pkg.RowNorm("layer", rand(rng, 256, "f16"), rand(rng, 256, "f16"))
    whole = weights.linear(x, pre=norm)
    idx = torch.arange(rows, dtype=torch.int32, device="cuda").roll(-7)
    for m in (0, 1, 100, rows):
        some = weights.linear(x, pre=norm, idx=idx, count=torch.tensor([m], dtype=torch.int32, device="cuda"))
        assert torch.equal(some[:m], whole[idx[:m].long()]), m


# ---- refusals ---------------------------------------------------------------------------------------------------------
def test_no_rows(ctx):
    e = torch.empty(0, 48, device="cuda")
    y, z, q, qs = ctx.rows_norm(e, e, y=True, z=True, q=True)
    assert y.shape == (0, 48) and z.shape == (0, 48) and q.shape == (0, 48)
    w, ws = q_weights(np.random.default_rng(0), 48, 9)
    weights = pkg.RowWeights(ctx, w, scale=ws)
    assert weights.linear(e).shape == (0, 9) and weights.matmul(q, qs).shape == (0, 9)
    ctx.sync()


def test_python_refusals(ctx):
    x = torch.zeros(4, 32, device="cuda")
    w, ws = q_weights(np.random.default_rng(0), 32, 8)
    weights = pkg.RowWeights(ctx, w, scale=ws)
    idx = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: ctx.rows_norm(), lambda: ctx.rows_norm(x.double(), z=True), lambda: ctx.rows_norm(x, x[:, :16], y=True),
                lambda: ctx.rows_norm(x, x[:2], y=True), lambda: ctx.rows_norm(x, x.half(), y=True), lambda: ctx.rows_norm(x.t().contiguous().t(), z=True),
                lambda: ctx.rows_norm(x.cpu(), z=True), lambda: ctx.rows_norm(x, z=True, idx=idx.long()), lambda: ctx.rows_norm(x, z=True, count=idx),
                lambda: ctx.rows_norm(x, x, gate=x[:1], gate_rows=2, y=True), lambda: ctx.rows_norm(x, pre=pkg.RowNorm("rms", ws), z=True),
                lambda: ctx.rows_norm(x, q=torch.zeros(4, 32, device="cuda")), lambda: ctx.rows_norm(x[:1].expand(4, 32), z=True),
                lambda: pkg.RowWeights(ctx, w), lambda: pkg.RowWeights(ctx, w.float(), scale=ws), lambda: pkg.RowWeights(ctx, w, scale=ws[:4]),
                lambda: pkg.RowWeights(ctx, w.t(), scale=ws), lambda: pkg.RowWeights(ctx, torch.zeros(65537, 4, device="cuda")),
                lambda: pkg.RowWeights(ctx, w, scale=ws, bias=ws[:4]), lambda: weights.linear(x[:, :16]), lambda: weights.linear(x, idx=idx.float()),
                lambda: weights.matmul(x, ws), lambda: weights.matmul(x.to(torch.int8), ws[:2]), lambda: weights.linear(x, out=x),
                lambda: pkg.RowWeights(ctx, w, scale=ws, bias=ws.half()).linear(x)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(KeyError):
        pkg.RowNorm("batch")
    for bad, status in ((lambda: ctx.rows_norm(x), 1), (lambda: ctx.rows_norm(x, gate=x, y=None, z=True), 1), (lambda: ctx.rows_norm(x, post=pkg.RowNorm("rms"), z=True), 1),
                        (lambda: ctx.rows_norm(x, pre=pkg.RowNorm("rms", eps=-1.0), z=True), 1), (lambda: ctx.rows_norm(x, x, scale=float("nan"), y=True), 1),
                        (lambda: ctx.rows_norm(x, x, gate=x, gate_rows=-1, y=True), 1), (lambda: ctx.rows_norm(torch.zeros(1, 32769, device="cuda"), z=True), 7),
                        (lambda: ctx.rows_norm(x, q=torch.zeros(4, 40, dtype=torch.int8, device="cuda")[:, :32]), 1),
                        (lambda: weights.matmul(torch.zeros(5, 33, dtype=torch.int8, device="cuda")[:4, 1:], ws), 1)):
        with pytest.raises(pkg.DcnnError) as e:
            bad()
        assert e.value.status == status, e.value


def test_in_place_needs_one_spacing(ctx):
    """Rows that lie elsewhere in y than in x would be written over before they are read."""
    base = torch.ones(8, 32, device="cuda")
    x, h = base[:4], torch.ones(4, 32, device="cuda")
    with pytest.raises(pkg.DcnnError) as e:
        ctx.rows_norm(x, h, y=base[::2])
    assert e.value.status == 2, e.value
    ctx.rows_norm(x[:1], h[:1], y=base[::2][:1])               # (one row lies where it lies)
    ctx.rows_norm(base[::2], h, y=base[::2])
    ctx.sync()
    want = torch.ones(8, 32)
    want[::2] += 1
    want[0] += 1
    assert torch.equal(base.cpu(), want)


def test_outputs_in_the_place_of_inputs_are_refused(ctx):
    x, h, y, z = (torch.zeros(8, 32, device="cuda") for _ in range(4))
    weights = pkg.RowWeights(ctx, torch.ones(32, 32, device="cuda"))
    for bad in (lambda: ctx.rows_norm(x, h, y=h), lambda: ctx.rows_norm(x, h, z=h), lambda: ctx.rows_norm(x, h, z=x), lambda: ctx.rows_norm(x, h, y=y, z=y),
                lambda: ctx.rows_norm(x, z=x), lambda: ctx.rows_norm(None, h, y=h), lambda: weights.linear(x, out=x)):
        with pytest.raises(pkg.DcnnError) as e:
            bad()
        assert e.value.status == 1, e.value
    ctx.rows_norm(x, x, y=y, z=z)                              # (inputs may be one)
    ctx.rows_norm(x, h, y=x, z=z)
    ctx.sync()


def test_c_refusals(ctx):
    """The C entry points check what the binding would not let through; nothing is launched."""
    import ctypes as C
    from paper_2203_03996_amd.binding import RowsMatmulArgs, RowsNormArgs
    lib = ctx.lib
    x = torch.zeros(4, 64, device="cuda")
    q = torch.zeros(4, 64, dtype=torch.int8, device="cuda")
    out = torch.full((4, 64), 3.0, device="cuda")
    p, o = x.data_ptr(), out.data_ptr()

    def norm(**kw):
        a = RowsNormArgs(c=64, x=p, z=o, ldx=64, ldz=64, scale=1.0)
        a.rows = a.map_rows = 4
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.dcnn_rows_norm(ctx.handle, C.byref(a))
    assert norm(dtype=3) == 3 and norm(dtype=-1) == 3 and norm(dtype=9) == 3
    assert norm(c=0) == 1 and norm(c=32769) == 7 and norm(rows=-1) == 1 and norm(rows=1 << 31) == 1 and norm(rows=5) == 2 and norm(map_rows=-1) == 1
    assert norm(ldx=63) == 2 and norm(ldz=1 << 31) == 7 and norm(x=None) == 1 and norm(z=None) == 1 and norm(x=p + 2) == 1 and norm(idx=p + 1) == 1 and norm(count=p + 2) == 1
    assert norm(y=o, ldy=64) == 1 and norm(gate=p) == 1 and norm(q=q.data_ptr(), ldq=64) == 1 and norm(q=q.data_ptr() + 8, q_scale=p, ldq=64) == 1
    assert norm(q=q.data_ptr(), q_scale=p, ldq=72) == 1 and norm(q=q.data_ptr(), q_scale=p, ldq=48) == 2 and norm(gate_rows=-1) == 1
    assert lib.dcnn_rows_norm(None, None) == 1 and lib.dcnn_rows_norm(ctx.handle, None) == 1

    w, ws = q_weights(np.random.default_rng(0), 64, 64)
    weights = pkg.RowWeights(ctx, w, scale=ws)
    nbytes = lib.dcnn_rows_weights_bytes(64, 64)
    packed = weights.packed.data_ptr()
    assert lib.dcnn_rows_pack(ctx.handle, 0, 64, 64, p, 64, None, packed, nbytes - 1) == 5
    assert lib.dcnn_rows_pack(ctx.handle, 0, 64, 64, p, 63, None, packed, nbytes) == 2
    assert lib.dcnn_rows_pack(ctx.handle, 0, 64, 64, p, 64, p, packed, nbytes) == 1
    assert lib.dcnn_rows_pack(ctx.handle, 3, 64, 64, p, 64, None, packed, nbytes) == 1
    assert lib.dcnn_rows_pack(ctx.handle, 4, 64, 64, p, 64, None, packed, nbytes) == 3
    assert lib.dcnn_rows_pack(ctx.handle, 0, 65537, 64, p, 64, None, packed, 1 << 40) == 1
    assert lib.dcnn_rows_pack(ctx.handle, 0, 64, 64, p, 64, None, packed + 16, nbytes) == 1
    assert lib.dcnn_rows_pack(ctx.handle, 0, 64, 64, None, 64, None, packed, nbytes) == 1
    assert lib.dcnn_rows_pack(None, 0, 64, 64, p, 64, None, packed, nbytes) == 1

    scratch = torch.zeros(lib.dcnn_rows_scratch_bytes(4, 64, 64, 1) + 256, dtype=torch.uint8, device="cuda")

    def product(linear, **kw):
        a = RowsMatmulArgs(k=64, n=64, packed=packed, y=o, ldy=64, scratch=scratch.data_ptr(), scratch_bytes=scratch.numel())
        a.rows = a.map_rows = 4
        if linear:
            a.x, a.ldx = p, 64
        else:
            a.q, a.q_scale, a.ldq = q.data_ptr(), ws.data_ptr(), 64
        for k, v in kw.items():
            setattr(a, k, v)
        return (lib.dcnn_rows_linear if linear else lib.dcnn_rows_matmul)(ctx.handle, C.byref(a))
    for linear in (False, True):
        assert product(linear, dtype=3) == 3 and product(linear, act=3) == 1 and product(linear, k=0) == 1 and product(linear, n=0) == 1 and product(linear, n=1 << 25) == 1
        assert product(linear, rows=-1) == 1 and product(linear, packed=None) == 1 and product(linear, packed=packed + 16) == 1 and product(linear, y=None) == 1
        assert product(linear, ldy=63) == 2 and product(linear, y=o + 2) == 1 and product(linear, bias=p + 1) == 1 and product(linear, count=p + 1) == 1
    assert product(False, x=p) == 1 and product(False, idx=p) == 1 and product(False, q=None) == 1 and product(False, q_scale=None) == 1
    assert product(False, ldq=60) == 1 and product(False, ldq=48) == 2 and product(False, q=q.data_ptr() + 4) == 1
    assert product(True, q=q.data_ptr()) == 1 and product(True, x=None) == 1 and product(True, ldx=60) == 2 and product(True, rows=5) == 2
    assert product(True, scratch_bytes=64) == 5 and product(False, scratch_bytes=64) == 5 and product(True, scratch=None) == 1 and product(True, scratch=scratch.data_ptr() + 16) == 1
    assert product(True, k=40000, packed=packed) == 7
    for call in (lib.dcnn_rows_linear, lib.dcnn_rows_matmul):
        assert call(None, None) == 1 and call(ctx.handle, None) == 1
    ctx.sync()
    assert (np64(out) == 3.0).all(), "a refused call wrote something"


# ---- blocks on a network's updates ------------------------------------------------------------------------------------
def block64(x, up, down, ub, db, pre, post, gate, scale):
    """A block in 64 bits, quantised where the operators quantise."""
    quant = lambda v: (np.rint(v * 127 / np.abs(v).max(-1, keepdims=True)), np.abs(v).max(-1, keepdims=True) / 127)  # noqa: E731
    wq = lambda w: tuple(a.T for a in quant(w.T))  # noqa: E731
    q, s = quant(norm64(x, *pre)[0])
    w, ws = wq(up)
    hidden = np.maximum((q @ w) * s * ws + ub, 0)
    q, s = quant(hidden)
    w, ws = wq(down)
    return x + scale * gate * norm64((q @ w) * s * ws + db, *post)[0]


def test_block_follows_its_formula(ctx):
    """Between the two products the hidden rows are rounded to fp16, which moves an 8-bit value by one step now and then;
    that is 1/127 of a row's largest value, at most, times a weight.  Over `hidden` of them the steps add up like a random walk."""
    rng = np.random.default_rng(8)
    c, hidden, px = 96, 200, 300
    t = {k: rand(rng, s, "f16", sc, m) for k, (s, sc, m) in {"up": ((c, hidden), c ** -0.5, 0), "down": ((hidden, c), hidden ** -0.5, 0), "ub": (hidden, 0.1, 0), "db": (c, 0.1, 0),
                                                             "w1": (c, 0.1, 1), "b1": (c, 0.1, 0), "w2": (c, 0.1, 1), "gate": (c, 0.1, 0.5), "x": ((px, c), 1, 0)}.items()}
    block = pkg.RowBlock(ctx, t["up"], t["down"], t["ub"], t["db"], pre=pkg.RowNorm("layer", t["w1"], t["b1"]), post=pkg.RowNorm("rms", t["w2"]), gate=t["gate"], scale=0.5)
    y = block.step(t["x"], torch.zeros_like(t["x"]))
    ctx.sync()
    v = {k: np64(a) for k, a in t.items()}
    want = block64(v["x"], v["up"], v["down"], v["ub"], v["db"], ("layer", v["w1"], v["b1"], 1e-5), ("rms", v["w2"], None, 1e-5), v["gate"], 0.5)
    # the block's branch is of the size of `gate`; a hidden value of 127 steps is off by half of fp16's spacing there, 127 * 2^-11 of a step at most,
    # so about one in sixteen moves a step: sqrt(hidden / 16) steps of 1 / 127 of the largest hidden value (about 3 of its rms), relative to sqrt(hidden) rms
    off = np.abs(np64(y) - want).max()
    assert off <= 0.5 * 1.0 * (6 * 3 / 127 / 4) + 2.0 ** -11 * np.abs(want).max(), off


def test_blocks_on_the_flagged_pixels_of_a_network():
    import examples.video_tokens as example
    found = example.run(streams=2, size=32, hidden=192, frames=5)
    assert len(found) == 4 and all(0 < n < px for n, px, _, _ in found)


def test_token_stack_wants_its_first_frame(ctx):
    stack = pkg.TokenStack([pkg.RowBlock(ctx, torch.ones(8, 16, device="cuda"), torch.ones(16, 8, device="cuda"))])
    with pytest.raises(ValueError):
        stack.step(torch.ones(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        pkg.RowBlock(ctx, torch.ones(8, 16, device="cuda"), torch.ones(8, 16, device="cuda"))
