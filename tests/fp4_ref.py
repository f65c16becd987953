"""4-bit rows from their definition in float64 (torch, any device): what quantize_fp4 has to give bit
for bit, and what its bytes stand for."""
import torch

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
E4M3 = tuple(m / 512 for m in range(8)) + tuple((8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8))[:-1]


def nearest(y, grid):
    """Index of the number of the grid nearest to y >= 0, the even one of two; y beyond its end: the end."""
    g = torch.tensor(grid, dtype=torch.float64, device=y.device)
    hi = torch.searchsorted(g, y.contiguous()).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    below, above = y - g[lo], g[hi] - y
    return torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def quantize(x):
    """(codes uint8 [M, d], scales as e4m3 bytes [M, ceil(d / 16)], row scales float64 [M]) of x [M, d]."""
    v = x.double()
    M, d = v.shape
    top = v.abs().amax(1)
    bad = ~torch.isfinite(top)
    v = torch.where(bad[:, None], 0.0, v)
    top = torch.where(bad, 0.0, top)
    r = torch.full_like(top, 2.0 ** -126)
    for _ in range(300):                       # the least power of two with top <= 2688 r
        r = torch.where(top > 2688 * r, 2 * r, r)
    v = torch.nn.functional.pad(v, (0, -d % 16)).unflatten(1, (-1, 16)) / r[:, None, None]
    sb = nearest(v.abs().amax(-1) / 6, E4M3)
    s = torch.tensor(E4M3, dtype=torch.float64, device=x.device)[sb].unsqueeze(-1)
    c = torch.where(s > 0, nearest((v / torch.where(s > 0, s, 1.0)).abs(), E2M1) + 8 * torch.signbit(v), 0)
    r = torch.where(bad, float("nan"), torch.where(top > 0, r, 0.0))
    return c.flatten(1)[:, :d].to(torch.uint8), sb.to(torch.uint8), r


def bytes_of(c, sb):
    """The library's bytes: codes [M, ceil(d / 2)], scales [ceil(M / 128), ceil(d / 64), 512] (0 in rows behind M)."""
    c = torch.nn.functional.pad(c, (0, c.shape[1] % 2)).unflatten(1, (-1, 2))
    M, B = sb.shape
    blocks = torch.zeros(-(-M // 128), -(-B // 4), 512, dtype=torch.uint8, device=c.device)
    m, b = torch.arange(M, device=c.device)[:, None], torch.arange(B, device=c.device)[None]
    blocks[m // 128, b // 4, 16 * (m % 32) + 4 * (m % 128 // 32) + b % 4] = sb
    return c[..., 0] | (c[..., 1] << 4), blocks


def values(q, blocks, scale, d):
    """float64 [M, d] that the bytes stand for."""
    M = q.shape[0]
    n = torch.stack([q & 15, q >> 4], -1).flatten(1)[:, :d].long()
    m, b = torch.arange(M, device=q.device)[:, None], (torch.arange(d, device=q.device) // 16)[None]
    sb = blocks[m // 128, b // 4, 16 * (m % 32) + 4 * (m % 128 // 32) + b % 4].long()
    table = lambda v: torch.tensor(v, dtype=torch.float64, device=q.device)
    e4m3 = table(E4M3 + (float("nan"),))
    s = torch.where(sb < 128, 1.0, -1.0) * e4m3[sb & 127]
    return table(E2M1 + tuple(-v for v in E2M1))[n] * s * scale.double()[:, None]


def untouched(blocks, rows):
    """Mask of the bytes of blocks that no row below `rows` has."""
    i = torch.arange(512, device=blocks.device)
    m = (i // 16) + 32 * (i % 16 // 4)
    t = torch.arange(blocks.shape[0], device=blocks.device)[:, None, None]
    return (128 * t + m[None, None] >= rows).expand_as(blocks)
