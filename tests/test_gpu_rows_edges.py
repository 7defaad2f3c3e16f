"""Row operators at the edges of what they take: schedules of few K-tiles, parameters that move, outputs that are too short or lie elsewhere
than they should, the longest calls.  Tolerances as in test_gpu_rows.py."""
import numpy as np
import pytest
import torch

import paper_2203_03996_amd as pkg
from tests.test_gpu_rows import TYPES, U32, close, ctx, np64, q_rows, q_weights, rand  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- workgroups with few K-tiles --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows,n", [(64, 1024), (130, 256), (700, 300), (2048, 1536), (1000, 4100), (4000, 3000)])
@pytest.mark.parametrize("k", [1, 128, 129, 200, 256, 257, 384, 385])
def test_product_of_few_k_tiles(ctx, dt, rows, n, k):  # noqa: F811
    """One to four K-tiles to a tile, where two and three of them are copied ahead; one tile to a workgroup and several."""
    product_at_some_rows(ctx, dt, rows, k, n)


@pytest.mark.parametrize("rows,n", [(64, 1024), (30, 600), (128, 512)])
@pytest.mark.parametrize("k", [8193, 8256, 8320, 8321, 9216, 9217, 16385])
def test_product_whose_last_part_is_short(ctx, rows, n, k):  # noqa: F811
    """A k that workgroups share, of which the last one's part is one, two or three K-tiles."""
    product_at_some_rows(ctx, "f32", rows, k, n)


def product_at_some_rows(ctx, dt, rows, k, n):  # noqa: F811
    rng = np.random.default_rng([rows, k, n])
    q, qs = q_rows(rng, rows, k)
    w, ws = q_weights(rng, k, n)
    bias = rand(rng, n, dt)
    y = pkg.RowWeights(ctx, w, scale=ws, bias=bias).matmul(q, qs, dtype=TYPES[dt][0])
    ctx.sync()
    at = torch.from_numpy(np.unique(np.concatenate([np.arange(min(rows, 70)), rng.integers(0, rows, 130), np.arange(max(0, rows - 70), rows)]))).cuda()
    s = (q[at].double() @ w.double()) * qs[at].double()[:, None] * ws.double()          # (whole numbers below 2^53 before the scales)
    close(y[at], np64(s + bias.double()), dt, np64(4 * U32 * (s.abs() + bias.double().abs())), f"{dt} {rows}x{k}x{n}")


# ---- parameters that move ---------------------------------------------------------------------------------------------
def test_parameters_are_read_where_they_lie_at_each_call(ctx):  # noqa: F811
    """Norms, biases and gates of a module whose storage is swapped between calls."""
    c, n, rows = 64, 96, 40
    rng = np.random.default_rng(1)
    layer = torch.nn.LayerNorm(c).cuda()
    bias = torch.nn.Parameter(torch.zeros(n, device="cuda"), requires_grad=False)
    gate = torch.nn.Parameter(torch.ones(c, device="cuda"), requires_grad=False)
    norm = pkg.RowNorm("layer", layer.weight, layer.bias)
    w, ws = q_weights(rng, c, n)
    weights = pkg.RowWeights(ctx, w, scale=ws, bias=bias)
    up, down = rand(rng, (c, n), "f32"), rand(rng, (n, c), "f32")
    block = pkg.RowBlock(ctx, up, down, up_bias=bias, pre=norm, gate=gate)
    for dt in ("f32", "f16", "f32", "bf16"):
        for t in (*layer.parameters(), bias, gate):
            t.data = rand(rng, t.shape, dt, 0.3, 0.5)              # (what lay there before is freed)
        x = rand(rng, (rows, c), dt)
        fresh = pkg.RowNorm("layer", layer.weight.data.clone(), layer.bias.data.clone())
        fresh_weights = pkg.RowWeights(ctx, w, scale=ws, bias=bias.data.clone())
        fresh_block = pkg.RowBlock(ctx, up, down, up_bias=bias.data.clone(), pre=fresh, gate=gate.data.clone())
        got, want = weights.linear(x, pre=norm), fresh_weights.linear(x, pre=fresh)
        z, zw = ctx.rows_norm(x, pre=norm, z=True)[1], ctx.rows_norm(x, pre=fresh, z=True)[1]
        y, yw = block.step(x, torch.empty_like(x)), fresh_block.step(x, torch.empty_like(x))
        ctx.sync()
        assert torch.equal(got, want) and torch.equal(z, zw) and torch.equal(y, yw), dt
        for other in set(TYPES) - {dt}:
            xo = x.to(TYPES[other][0])
            for bad in (lambda: weights.linear(xo), lambda: ctx.rows_norm(xo, pre=norm, z=True), lambda: weights.linear(xo, pre=fresh)):
                with pytest.raises(ValueError):
                    bad()
    bias.data = torch.zeros(n + 1, device="cuda")
    with pytest.raises(ValueError):
        weights.linear(rand(rng, (rows, c), "f32"))
    bias.data = torch.zeros(n)                                     # not on the GPU
    with pytest.raises(ValueError):
        weights.linear(rand(rng, (rows, c), "f32"))


# ---- scratch ----------------------------------------------------------------------------------------------------------
def test_scratch_made_in_a_capture_while_torch_is_on_another_stream():
    """The context's stream is captured, torch is on a stream that has forked from it: scratch that the graph clears is the graph's alone."""
    rng = np.random.default_rng(29)
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = pkg.Context(0)  # noqa: F811
    k, n, rows = 4096, 128, 160                                     # (workgroups that share a tile count themselves in the scratch)
    w, ws = q_weights(rng, k, n)
    x = rand(rng, (400, k), "f16")
    torch.cuda.synchronize()
    weights = pkg.RowWeights(ctx, w, scale=ws)
    want = pkg.RowWeights(ctx, w, scale=ws).linear(x)
    out = torch.zeros(rows, n, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        assert ctx.capturing()
        other.wait_stream(stream)
        with torch.cuda.stream(other):
            assert ctx.capturing()
            weights.linear(x[:rows], out=out)
        stream.wait_stream(other)
    assert weights._grown is None and not ctx.capturing()          # (nothing has cleared what the capture made)
    for eager in (rows, 400, 100):
        with torch.cuda.stream(other):
            got = weights.linear(x[:eager])
        ctx.sync()
        assert torch.equal(got, want[:eager]), eager
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[:rows]), eager
        out.zero_()
        torch.cuda.synchronize()


# ---- matrices that are too short --------------------------------------------------------------------------------------
def test_matrices_with_too_few_rows_are_refused(ctx):  # noqa: F811
    """Every row of a call without a count is wanted: none is left out because another matrix has no room for it."""
    rng = np.random.default_rng(3)
    x, h, y = rand(rng, (8, 32), "f32"), rand(rng, (8, 32), "f32"), torch.full((8, 32), 7.0, device="cuda")
    short = torch.full((4, 32), 7.0, device="cuda")
    q, qs = torch.zeros(4, 32, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    w, ws = q_weights(rng, 32, 32)
    weights = pkg.RowWeights(ctx, w, scale=ws)
    rows, scales = ctx.rows_quantize(x)
    idx = torch.arange(8, dtype=torch.int32, device="cuda")
    for listed in (None, idx):
        for bad in (lambda: ctx.rows_norm(x, h, y=y, z=short, idx=listed), lambda: ctx.rows_norm(x, h, y=y, q=q, q_scale=qs, idx=listed),
                    lambda: ctx.rows_norm(x, h[:4], y=y, idx=listed), lambda: ctx.rows_norm(x, z=short, idx=listed), lambda: weights.linear(x, out=short, idx=listed),
                    lambda: weights.matmul(rows, scales, dtype=torch.float32, out=short)):
            with pytest.raises(ValueError, match="rows"):
                bad()
    ctx.sync()
    assert (np64(y) == 7.0).all() and (np64(short) == 7.0).all(), "a refused call wrote something"


@pytest.mark.parametrize("count,m", [(3, 3), (4, 4), (9, 4)])
def test_a_count_goes_with_matrices_of_less_room(ctx, count, m):  # noqa: F811
    """A list has room for the whole map and the matrices for the rows that there are: they are the call's room."""
    rng = np.random.default_rng(3)
    x, h = rand(rng, (20, 32), "f32"), rand(rng, (4, 32), "f32")
    w, ws = q_weights(rng, 32, 48)
    weights = pkg.RowWeights(ctx, w, scale=ws)
    at = torch.from_numpy(rng.permutation(20).astype(np.int32)).cuda()
    c = torch.tensor([count], dtype=torch.int32, device="cuda")
    y, z, out, two = (torch.full(s, 7.0, device="cuda") for s in ((20, 32), (4, 32), (4, 48), (4, 48)))
    q, qs = torch.zeros(4, 32, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    ctx.rows_norm(x, h, y=y, z=z, q=q, q_scale=qs, idx=at, count=c)
    weights.linear(x, out=out, idx=at, count=c)
    rows, scales = ctx.rows_quantize(x)
    weights.matmul(rows, scales, out=two, dtype=torch.float32, count=c)
    ctx.sync()
    i = at[:m].long()
    want = torch.full_like(y, 7.0)
    want[i] = x[i] + h[:m]
    assert torch.equal(y, want) and torch.equal(z[:m], want[i]) and (z[m:] == 7.0).all() and (q[m:] == 0).all()
    assert torch.equal(out[:m], weights.linear(x[i])) and (out[m:] == 7.0).all()
    assert torch.equal(two[:m], weights.linear(x[:m])) and (two[m:] == 7.0).all()


# ---- the longest calls ------------------------------------------------------------------------------------------------
def test_product_of_the_most_rows(ctx):  # noqa: F811
    """2^31 - 1 rows (34 GB of them): the last tile ends where 32 bits do."""
    rows, k = 0x7fffffff, 16
    rng = np.random.default_rng(31)
    w, ws = q_weights(rng, k, 1)
    ws.fill_(0.5)
    q, qs = torch.zeros(rows, k, dtype=torch.int8, device="cuda"), torch.full((rows,), 0.25, device="cuda")
    at = torch.tensor([0, 1, 127, 128, 1 << 30, rows - 300, rows - 256, rows - 129, rows - 128, rows - 127, rows - 2, rows - 1], device="cuda")
    q[at] = torch.from_numpy(rng.integers(-8, 9, (len(at), k), dtype=np.int8)).cuda()
    want = (q[at].double() @ w.double()) * 0.125 + 1.0             # (sums below 2^14, eighths: exact in fp32)
    weights = pkg.RowWeights(ctx, w, scale=ws, bias=torch.ones(1, device="cuda"))
    out = torch.empty(rows, 1, device="cuda")
    for count in (None, rows - 1, rows - 100, rows - 128, rows - 257, 3):
        out.fill_(-3.0)
        weights.matmul(q, qs, dtype=torch.float32, out=out, count=None if count is None else torch.tensor([count], dtype=torch.int32, device="cuda"))
        ctx.sync()
        n = rows if count is None else count
        here = at < n
        assert torch.equal(out[at[here]].double(), want[here]), count
        for lo in range(0, rows, 1 << 28):                         # rows of zeros are the bias, rows behind the count what they were
            part, end = out[lo:lo + (1 << 28)], max(0, min(n - lo, 1 << 28))
            assert int((part[:end] != 1.0).sum()) <= len(at) and bool((part[end:] == -3.0).all()), (count, lo)


def test_norm_of_the_most_rows(ctx):  # noqa: F811
    rows = 0x7fffffff
    x = torch.full((rows, 1), 0.5, dtype=torch.float16, device="cuda")
    x[rows - 1], x[rows - 2], x[0] = 3.0, 4.0, 5.0
    _, z, _, _ = ctx.rows_norm(x, z=True)
    ctx.sync()
    assert all(torch.equal(z[lo:lo + (1 << 28)], x[lo:lo + (1 << 28)]) for lo in range(0, rows, 1 << 28))


# ---- outputs that share bytes with what is read -----------------------------------------------------------------------
def test_outputs_that_reach_into_inputs_are_refused(ctx):  # noqa: F811
    """Not only at the same address: a row further on, in the middle, in the gate, in parameters, in one another."""
    buf = torch.full((40, 64), 2.0, device="cuda")
    x, h, z, y = buf[0:8], buf[8:16], buf[16:24], buf[24:32]
    whole = torch.ones(64, 64, device="cuda")
    weights = pkg.RowWeights(ctx, whole)
    idx = torch.arange(8, dtype=torch.int32, device="cuda")
    flat = buf.view(-1)
    q8 = torch.ones(40, 64, dtype=torch.int8, device="cuda")
    out8 = q8.view(torch.float32).view(-1)                         # the same bytes as floats
    scales = torch.ones(8, device="cuda")
    small = pkg.RowWeights(ctx, whole[:, :8].contiguous())
    bad = [lambda: ctx.rows_norm(x, h, y=buf[1:9]), lambda: ctx.rows_norm(x, h, y=buf[7:15]), lambda: ctx.rows_norm(x, h, y=flat[3:515].view(8, 64)),
           lambda: ctx.rows_norm(x, z=buf[1:9]), lambda: ctx.rows_norm(x, h, y=y, z=buf[25:33]), lambda: ctx.rows_norm(x, h, z=buf[9:17]),
           lambda: ctx.rows_norm(x, h, gate=y[:4], gate_rows=2, y=y), lambda: ctx.rows_norm(x, h, gate=y[5], y=y), lambda: ctx.rows_norm(x, h, gate=x, gate_rows=1, y=x),
           lambda: ctx.rows_norm(x, h, post=pkg.RowNorm("rms", y[3]), y=y), lambda: ctx.rows_norm(x, pre=pkg.RowNorm("layer", None, z[7]), z=z),
           lambda: ctx.rows_norm(x, q=buf.view(torch.int8).view(-1)[:8 * 64].view(8, 64), q_scale=scales), lambda: ctx.rows_norm(x, q=q8[:8], q_scale=flat[60:68]),
           lambda: ctx.rows_norm(x, h, y=y, q=q8[:8], q_scale=y.view(-1)[504:]), lambda: ctx.rows_norm(x, z=buf.view(torch.float32)[4:12], idx=idx),
           lambda: weights.linear(x, out=buf[1:9]), lambda: weights.linear(x, out=buf[6:14], idx=idx), lambda: weights.linear(x, pre=pkg.RowNorm("rms", z[1]), out=z),
           lambda: small.matmul(q8[:8], scales, dtype=torch.float32, out=out8[16:80].view(8, 8)),
           lambda: pkg.RowWeights(ctx, whole, bias=z[0]).linear(x, out=z)]
    for i, call in enumerate(bad):
        with pytest.raises(pkg.DcnnError) as e:
            call()
        assert e.value.status == 1 and "overlaps" in str(e.value), (i, e.value)
    need = ctx.lib.dcnn_rows_weights_bytes(64, 64)
    both = torch.full((need + 64 * 64 * 4,), 5, dtype=torch.uint8, device="cuda")
    at = both.data_ptr()
    assert ctx.lib.dcnn_rows_pack(ctx.handle, 0, 64, 64, at + need - 4, 64, None, at, need) == 1
    assert ctx.lib.dcnn_rows_pack(ctx.handle, 3, 64, 64, at + need, 64, at + need - 256, at, need) == 1
    ctx.sync()
    assert (buf == 2.0).all() and (q8 == 1).all() and (both == 5).all(), "a refused call wrote something"


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("c", [64, 61])
def test_matrices_between_the_columns_of_one_buffer(ctx, dt, c):  # noqa: F811
    """Views whose rows lie in each other's gaps share no byte: taken, and right."""
    rng = np.random.default_rng(c)
    rows = 50
    wide = rand(rng, (rows, 4 * c), dt)
    x, h, y, z = (wide[:, i * c:(i + 1) * c] for i in range(4))
    apart = [t.clone() for t in (x, h)]
    norm = pkg.RowNorm("rms", rand(rng, c, dt, 0.3, 1.0))
    want = ctx.rows_norm(*apart, post=norm, pre=norm, y=True, z=True)[:2]
    ctx.rows_norm(x, h, post=norm, pre=norm, y=y, z=z)
    assert torch.equal(y, want[0]) and torch.equal(z, want[1]) and torch.equal(x, apart[0]) and torch.equal(h, apart[1])
    weights = pkg.RowWeights(ctx, rand(rng, (c, c), dt))
    want = weights.linear(apart[0], pre=norm)
    weights.linear(x, pre=norm, out=z)
    assert torch.equal(z, want) and torch.equal(y, ctx.rows_norm(*apart, post=norm, y=True)[0])
    ctx.rows_norm(x, h, post=norm, y=x)                            # (in place, as before)
    assert torch.equal(x, y)


# ---- the context's GPU ------------------------------------------------------------------------------------------------
def test_weights_of_another_gpu_are_refused(ctx, monkeypatch):  # noqa: F811
    """(the context says that it is on another one)"""
    w, ws = q_weights(np.random.default_rng(0), 32, 8)
    x = torch.zeros(4, 32, device="cuda")
    weights = pkg.RowWeights(ctx, w, scale=ws)
    monkeypatch.setattr(ctx, "index", 1)
    for bad in (lambda: pkg.RowWeights(ctx, w, scale=ws), lambda: pkg.RowWeights(ctx, w.float()), lambda: weights.linear(x), lambda: ctx.rows_norm(x, z=True)):
        with pytest.raises(ValueError, match="GPU 1"):
            bad()


def test_threads_share_weights(ctx):  # noqa: F811
    """Linear calls of several sizes from several threads: each has its own rows' results."""
    import threading
    rng = np.random.default_rng(41)
    k, n = 512, 128
    w, ws = q_weights(rng, k, n)
    x = [rand(rng, (rows, k), "f16") for rows in (80, 300, 900, 2500)]
    want = [pkg.RowWeights(ctx, w, scale=ws).linear(t) for t in x]
    weights = pkg.RowWeights(ctx, w, scale=ws)
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        got = [weights.linear(x[i]) for _ in range(40)]
        torch.cuda.synchronize()
        wrong.extend(i for y in got if not torch.equal(y, want[i]))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


# ---- bits ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dt,ks", [("f16", (5, 77, 256, 300, 511, 512)), ("bf16", (8, 500, 512)), ("f32", (5, 77, 129, 255, 256))])
def test_rows_of_a_wave_have_the_same_bits_alone_and_among_many(ctx, dt, ks, kind):  # noqa: F811
    """Rows of up to 64 vectors of 16 bytes: normed by the kernel of one to four rows, by a tile's, or by the norm's own."""
    for k in ks:
        rng = np.random.default_rng(k)
        x = rand(rng, (700, k), dt, 1.5, 0.5)
        weights, norm = pkg.RowWeights(ctx, rand(rng, (k, 200), "f32")), pkg.RowNorm(kind, rand(rng, k, dt), rand(rng, k, dt))
        whole = weights.linear(x, pre=norm)
        q, qs = ctx.rows_quantize(x, pre=norm)
        assert torch.equal(whole, weights.matmul(q, qs, dtype=TYPES[dt][0])), k
        for r in (1, 2, 4, 40):
            assert torch.equal(weights.linear(x[:r], pre=norm), whole[:r]), (k, r)


@pytest.mark.parametrize("c", [1000, 2100, 4096])
def test_a_list_with_the_room_of_the_map_has_the_bits_of_the_map(ctx, c):  # noqa: F811
    """Long rows too: a list of the map's room takes the kernels that the map takes, or others with the same bits."""
    rng = np.random.default_rng(c)
    for px, m in ((4, 3), (60, 30), (900, 100)):
        x, h = rand(rng, (px, c), "f16"), rand(rng, (px, c), "f16")
        norm = pkg.RowNorm("layer", rand(rng, c, "f16"), rand(rng, c, "f16"))
        weights = pkg.RowWeights(ctx, rand(rng, (c, 300), "f16"))
        idx = torch.from_numpy(rng.permutation(px).astype(np.int32)).cuda()
        count = torch.tensor([m], dtype=torch.int32, device="cuda")
        at = idx[:m].long()
        assert torch.equal(weights.linear(x, pre=norm, idx=idx, count=count)[:m], weights.linear(x, pre=norm)[at])
        listed = ctx.rows_norm(x, h[idx.long()].contiguous(), post=norm, pre=norm, idx=idx, count=count, y=x.clone(), z=True)
        whole = ctx.rows_norm(x, h, post=norm, pre=norm, y=True, z=True)
        assert torch.equal(listed[0][at], whole[0][at]) and torch.equal(listed[1][:m], whole[1][at])
