"""Heads, the cache in 4 bits and attention at the edges of what their calls allow, against the plain forms in 64 bits (tolerances as in test_gpu_cache.py)."""
import pytest
import torch

import paper_2203_03996_amd as pkg
from tests import cache_plain as plain
from tests.test_gpu_cache import TYPES, U32, attention_block, check_append, close, ctx, ints, new_cache, norm_of, rand, seeded  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- rows without a token -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("style", ["halves", "pairs"])
def test_heads_of_rows_without_a_token_are_zeros_behind_any_norm(ctx, dt, kind, style):  # noqa: F811
    """Entries outside of the map and positions outside of the rotation's table; norms with weight and bias, an infinity and a NaN among the weights."""
    gen = seeded(31)
    dim, rows = 64, 9
    q, k = rand(gen, rows, 5 * dim, dt=dt), rand(gen, rows, 2 * dim, dt=dt)
    w, b = rand(gen, dim, dt=dt, scale=0.3, mean=1.0), rand(gen, dim, dt=dt, scale=0.3, mean=1.0)
    rotation = pkg.Rotation.of_positions(50, 32, style=style)
    idx = ints(3, -1, 0, 40, 7, 1 << 30, 8, 2, 5)                      # (of a map of 9 rows)
    pos = ints(4, 50, 6, -1, 8, 9, 2 ** 31 - 1, 11, 49)
    has = torch.tensor([i in range(9) and 0 <= int(pos[i]) < 50 for i in idx.tolist()], device="cuda")
    assert 2 < has.sum() < 7
    for broken in (False, True):
        if broken:
            w[3], w[40], w[41] = float("inf"), float("nan"), -float("inf")
        norm = pkg.RowNorm(kind, w, b, 1e-5)
        got = ctx.rows_heads(q, k, dim=dim, q_norm=norm, k_norm=norm, rotation=rotation, positions=pos, idx=idx)
        alone = ctx.rows_heads(q, dim=dim, q_norm=norm, idx=idx, count=ints(rows))         # (a list without a rotation: entries below zero alone)
        ctx.sync()
        for y, x in ((got[0], q), (got[1], k)):
            assert (y[~has] == 0).all(), f"{dt} {kind} {style}: rows without a token are {y[~has].abs().amax(1).tolist()}"
            if not broken:
                want, mag = plain.heads64(x[has], dim, kind, w, b, 1e-5, rotation.table, style, pos[idx.long()[has]])
                close(y[has], want, dt, 32 * U32 * mag, f"{dt} {kind} {style}")
        assert (alone[1] == 0).all() and (alone[3] != 0).any()


# ---- norms' weights that are no numbers -----------------------------------------------------------------------------
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("rot", [0, 32])
def test_an_infinite_weight_stays_in_its_channel_where_nothing_turns(ctx, dt, style, rot):  # noqa: F811
    gen = seeded(33)
    dim, rows = 64, 5
    q = rand(gen, rows, 2 * dim, dt=dt) + 3.0
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    rotation = pkg.Rotation.of_positions(rows, rot, style=style) if rot else None
    for kind in ("rms", "layer"):
        w, b = rand(gen, dim, dt=dt, scale=0.3, mean=1.0), rand(gen, dim, dt=dt, scale=0.3)
        w[40], w[55], b[50] = float("inf"), float("nan"), -float("inf")
        got = ctx.rows_heads(q, dim=dim, q_norm=pkg.RowNorm(kind, w, b, 1e-5), rotation=rotation, positions=pos)
        ctx.sync()
        want, mag = plain.heads64(q, dim, kind, w, b, 1e-5, rotation and rotation.table, style, pos)
        got = got.double().view(want.shape)
        assert torch.isinf(want[..., 40]).all() and torch.equal(torch.isinf(got), torch.isinf(want)) and torch.equal(got.sign().nan_to_num(7.0), want.sign().nan_to_num(7.0))
        sane = torch.ones(dim, dtype=torch.bool, device="cuda")
        sane[[40, 50, 55]] = False
        close(got[..., sane].contiguous(), want[..., sane], dt, 32 * U32 * mag[..., sane], f"{dt} {kind} {style}")


# ---- keys of any size -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_codes_of_keys_below_the_normal_range(ctx, dt):  # noqa: F811
    """Every border of two codes at the smallest scale and the one above it, the numbers next to them, and, by a rotation, numbers that only 64 bits tell from a border."""
    t, _, step = TYPES[dt]
    border = torch.tensor([0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 0.125, 0.375], dtype=torch.float64)
    rows = []
    for e in (-126, -125, -124):
        for nudge in (-1, 0, 1):
            for top in (0.0, 1.0, 6.0):
                block = torch.cat([border, -border]) * 2.0 ** e + nudge * step
                block = block * (block.abs() <= max(top, 1.0) * 2.0 ** e)                  # (blocks whose largest magnitude asks for less, and for this scale)
                rows.append(block)
    x = torch.stack(rows).to(t).cuda()
    n = len(x)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    cache = new_cache(ctx, 1, n, 1, 32, dt)
    check_append(ctx, cache, x, x.flip(0).contiguous(), torch.zeros_like(pos), pos, dt, "none", streams=torch.zeros_like(pos), positions=pos)
    # a - b sin, b + a sin: b a few steps, the sine so small that b sin and a sin are far below a step
    table = torch.ones(n, 16, 2, device="cuda")
    table[..., 1] = torch.where(torch.arange(n, device="cuda") % 2 == 0, 2.0 ** -20, -2.0 ** -20)[:, None]
    y = x.clone()
    y[:, 16:] = (torch.arange(16, device="cuda") - 8).to(t) * step
    rotation = pkg.Rotation(table)
    cache.append(y, x, rotation=rotation, streams=torch.zeros_like(pos), positions=pos)
    ctx.sync()
    c, s = plain.quantised(plain.heads64(y, 32, table=table, pos=pos)[0])
    at = (cache.pages[0, pos.long() // 16].long(), 0, slice(None), pos.long() % 16)
    assert torch.equal(cache.scales[at], s) and torch.equal(cache.codes[at], plain.pack(c))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_keys_that_are_finite_beyond_fp32_are_held_as_the_largest(ctx, dt):  # noqa: F811
    info = torch.finfo(TYPES[dt][0])
    gen = seeded(32)
    x = rand(gen, 6, 64, dt=dt)
    x = (x.double() * (info.max / x.double().abs().amax(1, keepdim=True))).clamp(-info.max, info.max).to(TYPES[dt][0])
    x[3], x[4, 40] = info.max, float("inf")
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    cache = new_cache(ctx, 1, 6, 1, 64, dt)
    zero = torch.zeros_like(pos)
    table = torch.full((6, 16, 2), 0.5 ** 0.5, device="cuda")
    w = torch.full((64,), info.max, dtype=TYPES[dt][0], device="cuda")
    for norm, p, turn in ((None, {}, table), (pkg.RowNorm("rms", w, None, 0.0), dict(kind="rms", w=w), None), (pkg.RowNorm("layer", w, w, 0.0), dict(kind="layer", w=w, b=w), table)):
        cache.append(x, x, norm=norm, rotation=None if turn is None else pkg.Rotation(turn), streams=zero, positions=pos)
        ctx.sync()
        want = plain.heads64(x, 64, table=turn, pos=pos, **p)[0]
        c, s = plain.quantised(want)
        at = (cache.pages[0, pos.long() // 16].long(), 0, slice(None), pos.long())
        assert torch.equal(cache.scales[at], s), f"{cache.scales[at].tolist()} and {s.tolist()}"
        assert torch.equal(cache.codes[at], plain.pack(c))


# ---- many rows ------------------------------------------------------------------------------------------------------
def test_heads_of_as_many_rows_as_there_may_be(ctx):  # noqa: F811
    """2^31 - 1 rows of one head, in place (128 GiB): numbers of rows next to the largest integer."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    rows, dim = 2 ** 31 - 1, 32
    if torch.cuda.mem_get_info()[0] < rows * dim * 2 + (4 << 30):
        pytest.skip("not enough memory for 2^31 - 1 rows")
    x = torch.empty(rows, dim, dtype=torch.float16, device="cuda")
    places = [slice(0, 200), slice(2 ** 30 - 100, 2 ** 30 + 100), slice(rows - 200, rows)]
    gen = seeded(36)
    before = []
    for p in places:
        x[p] = rand(gen, 200, dim, dt="f16", scale=2.0)
        before.append(x[p].clone())
    w = rand(gen, dim, dt="f16", scale=0.3, mean=1.0)
    try:
        ctx.rows_heads(x, dim=dim, q_norm=pkg.RowNorm("rms", w, None, 1e-5), q_out=x)
        ctx.sync()
        for p, was in zip(places, before):
            want, mag = plain.heads64(was, dim, "rms", w, None, 1e-5)
            close(x[p], want, "f16", 32 * U32 * mag, f"rows {p.start} on")
    finally:
        del x
        torch.cuda.empty_cache()


# ---- many weak tokens -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("gap", [8.0, 14.0, 17.5, 19.0])
def test_many_weak_tokens_behind_a_strong_one_count(ctx, rows, gap):  # noqa: F811
    """fp16: one token's weight is exp(gap) times each of 6000 others', whose sum matters.  A weight of 2^-39 of the largest is as good as zero for a row alone,
    one of 2^-32 for rows in tiles (the largest of these is 2^7 at least): half a step below fp16's normal range, for each token."""
    n, dim = 6001, 32
    cache = pkg.TokenCache(ctx, 1, n, 1, dim, dtype=torch.float16)
    v = torch.full((n, 1, dim), 6.0, dtype=torch.float64, device="cuda")
    k = torch.zeros((n, 1, dim), dtype=torch.float64, device="cuda")
    strong = 4500
    k[strong, 0, 0], v[strong] = 1.5, 0.0
    at, slot = torch.arange(n, device="cuda") // 64, torch.arange(n, device="cuda") % 64
    for which, x in ((0, k), (1, v)):
        c, s = plain.quantised(x, 13)
        cache.codes[at, which, :, slot], cache.scales[at, which, :, slot] = plain.pack(c), s
    q = torch.zeros(rows, dim, dtype=torch.float16, device="cuda")
    q[:, 0] = torch.linspace(gap, gap + 0.5, rows, device="cuda") / 1.5
    got = cache.attend(q, scale=1.0, streams=torch.zeros(rows, dtype=torch.int32, device="cuda"), positions=torch.zeros(rows, dtype=torch.int32, device="cuda"))
    ctx.sync()
    pages = torch.arange(cache.num_pages, device="cuda").view(1, -1)
    want, slack = plain.attend64(q, cache.codes, cache.scales, pages, 64, [0] * rows, [0] * rows, [n], 1.0, weight_u=2.0 ** -11, tiny=2.0 ** (-39 if rows == 1 else -32))
    close(got, want, "f16", slack, f"gap {gap}")


# ---- the largest numbers --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows", [1, 40])
def test_attend_largest_queries(ctx, rows):  # noqa: F811
    """fp32 queries up to the largest number meet keys as small: what is cut off them to 16 bits must not round up to infinity."""
    n, dim = 70, 32
    cache = pkg.TokenCache(ctx, 1, n, 1, dim, dtype=torch.float32)
    gen = seeded(34)
    k, v = rand(gen, n, dim) * 2.0 ** -126, rand(gen, n, dim)
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    cache.append(k, v, streams=zero, positions=torch.arange(n, dtype=torch.int32, device="cuda"))
    q = rand(gen, rows, dim)
    q[:, 0] = torch.finfo(torch.float32).max
    q[:, 1:3] *= 2.0 ** 100
    zero = zero[:1].expand(rows).contiguous()
    got = cache.attend(q, scale=0.5, streams=zero, positions=zero)
    ctx.sync()
    want, slack = plain.attend64(q, cache.codes, cache.scales, torch.arange(2, device="cuda").view(1, 2), 64, [0] * rows, [0] * rows, [n], 0.5, terms=3, weight_u=2.0 ** -24)
    close(got, want, "f32", slack, "largest queries")


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows", [1, 40])
def test_attend_of_one_token_is_what_the_cache_holds(ctx, dt, rows):  # noqa: F811
    """All codes at all scales whose numbers are in the type's normal range; each row sees one token."""
    first, last = {"f32": (4, 250), "f16": (127 - 13, 127 + 13), "bf16": (4, 250)}[dt]
    n, dim = last - first + 1, 32
    cache = pkg.TokenCache(ctx, 1, n, 1, dim, dtype=TYPES[dt][0], page=16)
    at, slot = torch.arange(n, device="cuda") // 16, torch.arange(n, device="cuda") % 16
    cache.codes[at, 1, 0, slot] = plain.pack(torch.arange(32, device="cuda") % 16).to(torch.uint8)
    cache.scales[at, 1, 0, slot, 0] = torch.arange(first, last + 1, dtype=torch.uint8, device="cuda")
    cache.scales[at, 0] = 127
    held = cache.read(streams=torch.zeros(n, dtype=torch.int32, device="cuda"), positions=torch.arange(n, dtype=torch.int32, device="cuda"))[1]
    q = rand(seeded(35), rows, dim, dt=dt)
    zero = torch.zeros(rows, dtype=torch.int32, device="cuda")
    for start in range(0, n, rows):
        pos = torch.arange(start, start + rows, dtype=torch.int32, device="cuda").clamp(max=n - 1)
        got = cache.attend(q, streams=zero, positions=pos, causal=True, window=1)
        ctx.sync()
        assert torch.equal(got, held[pos.long()]), f"{dt} tokens {start} on"


# ---- scratch --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("before", [0, 20, 300])
def test_graphs_keep_the_scratch_of_attention(before):
    """Captured without a call before it, behind a small one, behind one as large; then larger calls without the graph, whose scratch takes the place of the first."""
    stream = torch.cuda.Stream()
    heads, dim, n, rows = 2, 64, 3000, 40                              # (tokens of tiles are split: sums of parts in the scratch)
    gen = seeded(37)
    with torch.cuda.stream(stream):
        own = pkg.Context(0)
        cache = pkg.TokenCache(own, 1, n, heads, dim, dtype=torch.float16)
        zero = torch.zeros(n, dtype=torch.int32, device="cuda")
        pos = torch.arange(n, dtype=torch.int32, device="cuda")
        cache.append(*(rand(gen, n, heads * dim, dt="f16") for _ in range(2)), streams=zero, positions=pos)
        q = rand(gen, rows, 4 * dim, dt="f16")

        def call(rows, x=None):
            return cache.attend(rand(gen, rows, 4 * dim, dt="f16") if x is None else x, streams=zero[:rows], positions=pos[n - rows:], causal=True)
        if before:
            call(before)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            captured = [call(rows, q), call(rows, q)]
        for i in range(4):
            call(1000 if i == 0 else 2000 + 100 * i)
            stream.synchronize()
            torch.cuda.empty_cache()
            others = [torch.full((size,), 0x7f, dtype=torch.uint8, device="cuda") for size in (1 << 21, 1 << 22, 1 << 23)]      # (in the place of scratch that was let go)
            q.copy_(rand(gen, rows, 4 * dim, dt="f16"))
            graph.replay()
            stream.synchronize()
            got = [c.clone() for c in captured]
            assert all((o == 0x7f).all() for o in others), f"replay {i} has written where others' tensors lie"
            want = call(rows, q)
            stream.synchronize()
            assert all(torch.equal(g, want) for g in got), f"replay {i}"
            del others


def test_eager_attention_of_rising_sizes_holds_one_scratch(ctx):  # noqa: F811
    heads, dim, n = 2, 64, 3000
    cache = pkg.TokenCache(ctx, 1, n, heads, dim, dtype=torch.float16)
    gen = seeded(38)
    q = rand(gen, 600, 4 * dim, dt="f16")
    zero, pos = torch.zeros(600, dtype=torch.int32, device="cuda"), torch.arange(600, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    before, most = torch.cuda.memory_allocated(), 0
    for rows in range(7, 600):
        cache.attend(q[:rows], streams=zero[:rows], positions=pos[:rows], causal=True, out=out[:rows])
        most = max(most, ctx.lib.dcnn_cache_scratch_bytes(pkg.F16, rows, 4, heads, dim, 1, n))
    ctx.sync()
    assert torch.cuda.memory_allocated() - before <= most * 3 // 2 + (1 << 20)


# ---- together -------------------------------------------------------------------------------------------------------
def test_a_captured_block_replayed_with_other_numbers_of_pixels():
    """A block's step as a graph: replayed with other flagged pixels, from none to all, and eager steps between, it leaves the tokens and the cache that the eager step does."""
    streams, side, c = 3, 9, 96
    n = streams * side * side
    stream = torch.cuda.Stream()
    gen = seeded(39)
    with torch.cuda.stream(stream):
        own = pkg.Context(0)
        block = attention_block(own, gen, "f16", c, streams, side, 4, 2, 32)
        x, y = rand(gen, n, c, dt="f16"), torch.zeros(n, c, dtype=torch.float16, device="cuda")
        idx, count = torch.arange(n, dtype=torch.int32, device="cuda"), ints(n)
        block.step(x, y, idx, count)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            block.step(x, y, idx, count)
        for m in (40, 0, 1, n, 7, 200):
            at = torch.randperm(n, device="cuda", generator=gen)[:m].sort().values
            idx.fill_(1 << 30)
            idx[:m] = at.to(torch.int32)
            count.fill_(m)
            x[at] = rand(gen, m, c, dt="f16")
            before = y.clone(), block.cache.codes.clone(), block.cache.scales.clone()
            graph.replay()
            stream.synchronize()
            got = y.clone(), block.cache.codes.clone(), block.cache.scales.clone()
            for t, was in zip((y, block.cache.codes, block.cache.scales), before):
                t.copy_(was)
            block.step(x, y, idx, count)
            stream.synchronize()
            assert all(torch.equal(g, w) for g, w in zip(got, (y, block.cache.codes, block.cache.scales))), f"{m} pixels"
            rest = torch.ones(n, dtype=torch.bool, device="cuda")
            rest[at] = False
            assert torch.equal(y[rest], before[0][rest]) and (m == 0 or not torch.equal(y[at], before[0][at]))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [2, 90])
def test_a_cache_in_16_bits_serves_calls_in_fp32(ctx, dt, rows):  # noqa: F811
    """The memory is the same: appended in 16 bits, read and attended to in fp32, with weights kept."""
    n, heads, dim = 700, 2, 64
    gen = seeded(40)
    cache = pkg.TokenCache(ctx, 2, n, heads, dim, dtype=TYPES[dt][0])
    stream, pos = torch.arange(2, dtype=torch.int32, device="cuda").repeat_interleave(n), torch.arange(n, dtype=torch.int32, device="cuda").repeat(2)
    cache.append(*(rand(gen, 2 * n, heads * dim, dt=dt) for _ in range(2)), streams=stream, positions=pos)
    wide = pkg.TokenCache(ctx, 2, n, heads, dim, dtype=torch.float32, codes=cache.codes, scales=cache.scales)
    q = rand(gen, rows, 4 * dim, dt=dt).float()
    at = torch.randint(0, n, (rows,), dtype=torch.int32, device="cuda", generator=gen)
    of = torch.arange(rows, dtype=torch.int32, device="cuda") % 2
    got, held = wide.attend(q, streams=of, positions=at, causal=True), (cache.read(), wide.read())
    ctx.sync()
    assert all(torch.equal(a.float(), b) for a, b in zip(*held))
    want, slack = plain.attend64(q, cache.codes, cache.scales, torch.arange(22, device="cuda").view(2, 11), 64, of, at, [n, n], dim ** -0.5, True, 0, 3, 2.0 ** -24)
    close(got, want, "f32", slack, f"{dt} cache in fp32")
