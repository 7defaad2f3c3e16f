"""A video's tokens, kept up to date: a sparse network, and per-token blocks on the pixels of its output that changed.

    python examples/video_tokens.py [frames]

A bottleneck block runs on the changes of a synthetic clip and keeps its dense output; two blocks of row operators
(norm, 8-bit products, gated residual) recompute the tokens at the flagged pixels.  Every frame is compared with the
same blocks on the whole map, bit for bit, and both are timed.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2203_03996_amd as pkg  # noqa: E402
import workloads as wl  # noqa: E402


def make_blocks(ctx, c, hidden, n, seed=0):
    """`n` blocks of random weights over c channels."""
    rng = np.random.default_rng(seed)
    half = lambda *shape, scale=1.0, mean=0.0: torch.from_numpy((rng.standard_normal(shape) * scale + mean).astype(np.float16)).cuda()  # noqa: E731
    return [pkg.RowBlock(ctx, half(c, hidden, scale=c ** -0.5), half(hidden, c, scale=hidden ** -0.5), half(hidden, scale=0.1), half(c, scale=0.1),
                         pre=pkg.RowNorm("layer", half(c, scale=0.1, mean=1.0), half(c, scale=0.1)), post=pkg.RowNorm("rms", half(c, scale=0.1, mean=1.0)),
                         gate=half(c, scale=0.1, mean=0.5), scale=0.5) for _ in range(n)]


def flagged(ctx, update):
    """(list, count) of an update's pixels; a layer that keeps no list leaves a mask."""
    if update.idx is not None and update.count is not None:
        return update.idx, update.count
    _, idx, count = ctx.mask_compact(update.mask)
    return idx, count


def run(streams=2, size=64, hidden=512, frames=6, eps=0.3):
    """Per frame: (flagged pixels, pixels, microseconds on the flagged pixels, microseconds on the whole map)."""
    spec = wl.bottleneck_block(eps=eps, h=size, w=size, frames=frames)
    px = streams * size * size
    ctx = pkg.Context(px)
    net = pkg.Net(ctx, spec, wl.make_weights(spec, 1), streams, flags=3)
    clip = torch.from_numpy(wl.make_batch(spec["video"], 1, streams).astype(np.float16)).cuda()
    c = net.output().data.shape[-1]
    blocks = make_blocks(ctx, c, hidden, 2)
    sparse, dense = pkg.TokenStack(blocks), pkg.TokenStack(blocks)
    clock = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    found = []
    for t in range(frames):
        (net.step if t else net.init)(clip[t])
        update = net.output()
        if t == 0:
            tokens = sparse.init(update.data)
            whole = dense.init(update.data)
            ctx.sync()
        else:
            idx, count = flagged(ctx, update)
            clock[0].record()
            tokens = sparse.step(update.data, idx, count)
            clock[1].record()
            whole = dense.init(update.data)
            clock[2].record()
            ctx.sync()
            found.append((int(count), px, 1e3 * clock[0].elapsed_time(clock[1]), 1e3 * clock[1].elapsed_time(clock[2])))
        if not torch.equal(tokens, whole):
            raise AssertionError(f"frame {t}: tokens recomputed at flagged pixels differ from those of the whole map")
    return found


if __name__ == "__main__":
    for n, px, us, whole_us in run(streams=8, size=128, hidden=1024, frames=int(sys.argv[1]) if len(sys.argv) > 1 else 8):
        print(f"{n:7d} of {px} pixels flagged ({100 * n / px:4.1f} %): two blocks {us:7.1f} us, on the whole map {whole_us:7.1f} us")
