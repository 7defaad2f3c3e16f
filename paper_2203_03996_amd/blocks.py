"""Per-token blocks on the pixels of a map that changed (host logic only; the work runs in the library's row operators).

A block takes every pixel by itself -- norm, expansion, activation, projection, norm, gated residual -- so run on the
flagged pixels alone it gives what it would give on the whole map: the list and the count that a layer leaves with an
update are all it needs, and they never travel to the host.  (Bit for bit where the list has room for the map, as those
of layers have, or the channels of a row are at most 64 vectors of 16 bytes; a list of one to four longer rows is normed
by another kernel, whose sums are in another order.)  Its products run in 8-bit integers.

Between its two products a block holds the hidden rows of as many pixels as the list has room for, and each of its two
weights the 8-bit rows of as many.
"""
from __future__ import annotations

import torch

from .binding import Context, RowNorm, RowWeights


class RowBlock:
    """y = x + scale * gate * post(down(act(up(pre(x))))), token by token.

    up [c, hidden] and down [hidden, c]: floating-point weights (quantised here), or (int8 weights, float32 scales).
    pre, post: RowNorm or None.  gate: [c], or [groups, c] with gate_rows map rows to a group; None: 1."""

    def __init__(self, ctx: Context, up, down, up_bias=None, down_bias=None, act="relu", pre: RowNorm | None = None,
                 post: RowNorm | None = None, gate: torch.Tensor | None = None, gate_rows: int = 0, scale: float = 1.0):
        self.ctx, self.pre, self.post, self.gate, self.gate_rows, self.scale = ctx, pre, post, gate, gate_rows, scale
        (up, up_scale), (down, down_scale) = (w if isinstance(w, tuple) else (w, None) for w in (up, down))
        if up.shape != down.shape[::-1]:
            raise ValueError(f"up {tuple(up.shape)} and down {tuple(down.shape)} do not fit together")
        self.up = RowWeights(ctx, up, scale=up_scale, bias=up_bias, act=act)
        self.down = RowWeights(ctx, down, scale=down_scale, bias=down_bias)

    def step(self, x: torch.Tensor, y: torch.Tensor, idx: torch.Tensor | None = None, count: torch.Tensor | None = None):
        """Recomputes the tokens of y that idx (its first `count` entries) names, or all of them.  x and y are maps
        [..., c]; y may be x."""
        hidden = self.up.linear(x, pre=self.pre, idx=idx, count=count)
        out = self.down.linear(hidden, count=count)
        self.ctx.rows_norm(x, out, post=self.post, gate=self.gate, gate_rows=self.gate_rows, scale=self.scale, idx=idx, count=count, y=y)
        return y


class TokenStack:
    """Blocks one behind the other on an accumulated map, with the tokens of every block kept from frame to frame.

    init and step return the last block's tokens themselves, not a copy: the next step writes into them, and a caller that
    changes them changes what later frames start from."""

    def __init__(self, blocks: list[RowBlock]):
        self.blocks, self.maps = blocks, None

    def init(self, x: torch.Tensor) -> torch.Tensor:
        """First frame: every token."""
        self.maps = [self.blocks[0].ctx.empty(x.shape, x.dtype) for _ in self.blocks]
        return self._run(x, None, None)

    def step(self, x: torch.Tensor, idx: torch.Tensor, count: torch.Tensor) -> torch.Tensor:
        """Later frames: the tokens at the pixels where x has changed."""
        if self.maps is None or self.maps[0].shape != x.shape:
            raise ValueError("init with a map of this shape comes before step")
        return self._run(x, idx, count)

    def _run(self, x, idx, count):
        for block, y in zip(self.blocks, self.maps):
            x = block.step(x, y, idx, count)
        return x
