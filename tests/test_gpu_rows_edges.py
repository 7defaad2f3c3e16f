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
