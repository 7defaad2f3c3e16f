"""Plain forms, in 64 bits, of heads, the cache in 4 bits and attention over it (for the tests alone)."""
import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def heads64(x, dim, kind="none", w=None, b=None, eps=0.0, table=None, style="halves", pos=None):
    """(heads [rows, heads, dim] normed and rotated, magnitudes that meet in them)."""
    v = x.double().reshape(x.shape[0], -1, dim)
    mag = v.abs()
    if kind != "none":
        mean = v.mean(2, keepdim=True) if kind == "layer" else torch.zeros_like(v[..., :1])
        r = ((v - mean).square().mean(2, keepdim=True) + eps).rsqrt()
        w64 = 1.0 if w is None else w.double()
        b64 = 0.0 if b is None else b.double()
        mag = (mag + mean.abs()) * r * (1.0 if w is None else w64.abs()) + (0.0 if b is None else b64.abs())
        v = (v - mean) * r * w64 + b64
    if table is not None:
        rot = 2 * table.shape[1]
        c, s = (t[:, None] for t in table.double()[pos.long()].unbind(2))
        v, mag = v.clone(), mag.clone()
        first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if style == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
        a, d, ma, md = v[..., first].clone(), v[..., second].clone(), mag[..., first].clone(), mag[..., second].clone()
        v[..., first], v[..., second] = a * c - d * s, d * c + a * s
        mag[..., first], mag[..., second] = ma * c.abs() + md * s.abs(), md * c.abs() + ma * s.abs()
    return v, mag


def quantised(v, most=125):
    """(codes uint8 [..., n], scale bytes [..., n / 32]) of values in 64 bits: every candidate is looked at.  most: the largest exponent of a scale."""
    blocks = v.double().unflatten(-1, (-1, 32))
    amax = blocks.abs().amax(-1)
    broken = ~torch.isfinite(blocks).all(-1)
    e = torch.full(amax.shape, -126, dtype=torch.int64, device=v.device)
    for k in range(-125, most + 1):
        e[amax > 6.0 * 2.0 ** (k - 1)] = k
    u = torch.where(broken[..., None], torch.zeros_like(blocks), blocks * torch.exp2(-e[..., None].double()))  # (codes of a broken block are zeros)
    grid, u = GRID.to(v.device), u.clamp(-6.0, 6.0)
    off = (u.abs()[..., None] - grid).abs()
    best = off.amin(-1, keepdim=True)
    near = off == best
    even = torch.arange(8, device=v.device) % 2 == 0
    code = torch.where((near & even).any(-1), (near & even).to(torch.uint8).argmax(-1), near.to(torch.uint8).argmax(-1))
    code = torch.where(u < 0, code + 8, code) * (code > 0)     # (a zero is code 0)
    byte = torch.where(broken, torch.full_like(e, 255), e + 127)
    return code.flatten(-2).to(torch.uint8), byte.to(torch.uint8)


def values(codes, scales):
    """Numbers of packed codes [..., dim / 2] and scale bytes [..., dim / 32]."""
    nibble = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    v = GRID.to(codes.device)[nibble & 7] * (1.0 - 2.0 * (nibble >> 3))
    power = torch.exp2(scales.double() - 127.0)
    power[scales == 255] = float("nan")
    return v * power.repeat_interleave(32, -1)


def pack(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def stream_values(codes, scales, pages, stream, head, which, n, page):
    """(values [n, dim], which tokens have a page) of a stream's first n tokens."""
    per_stream = -(-n // page)
    numbers = pages[stream, :per_stream].long()
    ok = (numbers >= 0) & (numbers < codes.shape[0])
    at = torch.where(ok, numbers, torch.zeros_like(numbers))
    v = values(codes[at, which, head], scales[at, which, head]).flatten(0, 1)[:n]
    return v, ok.repeat_interleave(page)[:n]


def attend64(q, codes, scales, pages, page, stream, pos, lens, scale, causal=False, window=0, terms=1, weight_u=2.0 ** -11, tiny=0.0):
    """(outputs [rows, q_heads, dim], what they may be off before their last rounding).

    U = 2^-24.  A product of q and a key: its terms meet exactly and are added in fp32, (terms * dim + 8) U of their magnitudes; with scale and the
    subtraction of the maximum 8 U of the numbers that meet; both for a row's own key and its largest.  A weight is off by as much of itself, is rounded
    by `weight_u`, and where the type has a smallest number by `tiny` of the largest weight; sums of n weights and of n products, with a factor for each
    of at most n tiles, are good to (3 n + 64) U of the magnitudes."""
    U = 2.0 ** -24
    heads, dim = codes.shape[2], codes.shape[4] * 2
    rows, q_heads = q.shape[0], q.shape[1] // dim
    q64 = q.double().view(rows, q_heads, dim)
    out, slack = torch.zeros_like(q64), torch.zeros_like(q64)
    for r in range(rows):
        s = int(stream[r])
        if s < 0 or s >= pages.shape[0]:
            continue
        n = int(lens[s])
        lo, hi, p = 0, n, int(pos[r])
        if causal:
            hi = min(hi, p + 1)
        if window:
            lo, hi = max(lo, p - window + 1), min(hi, p + window)
        if hi <= lo:
            continue
        for h in range(heads):
            k, ok = stream_values(codes, scales, pages, s, h, 0, hi, page)
            v, _ = stream_values(codes, scales, pages, s, h, 1, hi, page)
            k, v, ok = k[lo:], v[lo:], ok[lo:]
            k, v = k[ok], v[ok]
            if not len(k):
                continue
            g = q_heads // heads
            qq = q64[r, h * g:(h + 1) * g]
            x = scale * (qq @ k.T)
            e = abs(scale) * (terms * dim + 8) * U * (qq.abs() @ k.abs().T) + 8 * U * x.abs()
            w = torch.softmax(x, 1)
            out[r, h * g:(h + 1) * g] = w @ v
            met = w @ v.abs()
            off = 2.0 * e.amax(1, keepdim=True) * 2.0 + weight_u + (3 * len(k) + 64) * U
            slack[r, h * g:(h + 1) * g] = off * met + tiny * w.amax(1, keepdim=True) * v.abs().sum(0)
    return out, slack
