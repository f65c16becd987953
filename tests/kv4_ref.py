"""The 4-bit cache in numpy, from its definition: codes, page bytes, and the attention
in 64 bits with a bound on the kernel's error."""
import numpy as np

DH = 128
_D = np.arange(DH)
_G, _R = _D // 32, _D % 32
K_BYTE = 16 * (_R // 8) + 4 * _G + (_R % 8) // 2
V_BYTE = 8 * (_R // 4) + 2 * _G + (_R % 4) // 2


def round_bf16(x):
    """float64 values >= 0 to the nearest bf16 value, ties to even (as float64)."""
    _, e = np.frexp(x)
    unit = np.ldexp(1.0, np.maximum(e, -125) - 8)
    return np.rint(x / unit) * unit


def quant(x):
    """Codes int [..., 128] and scales float64 [..., 4] of rows of real values."""
    g = x.astype(np.float64).reshape(*x.shape[:-1], 4, 32)
    top = np.abs(g).max(-1)
    with np.errstate(all="ignore"):
        s = np.where(np.isfinite(top), round_bf16(np.where(np.isfinite(top), top, 0.0) / 7.0), np.nan)
        c = np.rint(g / s[..., None]).clip(-7, 7)
        c = np.where((s > 0)[..., None], c, 0.0)
    return c.reshape(x.shape).astype(np.int64), s


def values(x):
    """What a row reads as after the cache."""
    c, s = quant(x)
    return c * np.repeat(s, 32, axis=-1)


def bf16_bits(s):
    return (np.where(np.isnan(s), np.float32("nan"), s).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def rows_bytes(x, byte):
    """(code bytes [..., 64], scale bytes [..., 8]) of rows."""
    c, s = quant(x)
    out = np.zeros((*x.shape[:-1], 64), np.uint8)
    for d in range(DH):
        out[..., byte[d]] |= ((c[..., d] + 8) << (4 * (d & 1))).astype(np.uint8)
    return out, np.ascontiguousarray(bf16_bits(s)).view(np.uint8)


def build_cache(ks, vs, page, rng, spare=2, junk=True):
    """Cache [pages, H, 144 page] and table [B, width] of per-sequence K, V [n, H, 128]; what
    is behind the tokens is junk (255: NaN scales), unused table entries name no page."""
    B, H = len(ks), ks[0].shape[1]
    need = [-(-len(k) // page) for k in ks]
    total = sum(need) + spare
    cache = np.full((total, H, 144 * page), 255 if junk else 0, np.uint8)
    ids = rng.permutation(total)
    table = np.full((B, max(1, max(need)) + 1), 10 ** 9, np.int32)
    at = 0
    for b, (k, v) in enumerate(zip(ks, vs)):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
        if len(k) == 0:
            continue
        parts = (*rows_bytes(k, K_BYTE), *rows_bytes(v, V_BYTE))
        for j in range(len(k)):
            p, o = table[b, j // page], j % page
            base = 0
            for part, size in zip(parts, (64, 8, 64, 8)):
                cache[p, :, base + o * size:base + (o + 1) * size] = part[j]
                base += size * page
    return cache, table


def attention(q, ks, vs, counts, causal, scale):
    """out and error bound (float64 [B, T, H, 128]) for q [B, T, H, 128] (the type's values as
    float64) over the cached values of ks, vs.

    The bound: scores are f32 sums of exact products (the tensor core adds u = c + 8 in
    0 .. 15 and starts at -8 sum q): with A = scale sum_g s_g 15 sum |q| every partial sum is
    below A, two MMAs and four multiply-adds a group cost at most (4 2^-23 + 6 2^-24) A <
    2^-20 A; weights are then off by 2 * 2^-20 A relative (numerator and sum), by 2^-11 for
    the rounding of p s to fp16, and by 2^-16 + n 2^-28 for exp2, the f32 sums of n terms
    (n / 64 steps of a warp, 2^-23 each) and the merges.  p s is held relative to 2^e 2^-9 with
    2^e at most the largest V scale: below fp16's normal range its rounding is absolute, half of
    2^-24 there, which with codes up to 7 is at most 7 smax 2^-34 for each of the n terms (a
    one-hot softmax shows it: the other tokens' shares are all there is of a channel whose
    code is 0)."""
    B, T, H, _ = q.shape
    out = np.zeros(q.shape)
    bound = np.zeros(q.shape)
    for b in range(B):
        n, c = len(ks[b]), min(counts[b], T)
        if n == 0:
            continue
        kc, s = quant(ks[b])
        k, v = kc * np.repeat(s, 32, -1), values(vs[b])
        G = H // k.shape[1]
        for h in range(H):
            kv = h // G
            qq = q[b, :c, h]
            x = qq @ k[:, kv].T * scale
            lim = (n - c + np.arange(c) + 1) if causal else np.full(c, n)
            x = np.where(np.arange(n)[None] < lim[:, None], x, -np.inf)
            m = x.max(-1, keepdims=True)
            p = np.exp(x - np.where(np.isfinite(m), m, 0.0))
            z = p.sum(-1, keepdims=True)
            p = p / np.where(z > 0, z, 1.0)
            out[b, :c, h] = p @ v[:, kv]
            absq = np.abs(qq).reshape(c, 4, 32).sum(-1)                # [c, 4]
            A = (absq @ s[:, kv].T * 15 * scale).max(-1, keepdims=True)
            rel = 2 * 2.0 ** -20 * A + 2.0 ** -11 + 2.0 ** -16 + n * 2.0 ** -28
            top = 7 * quant(vs[b])[1][:, kv].max()
            bound[b, :c, h] = np.where(lim[:, None] > 0, rel * (p @ np.abs(v[:, kv])) + n * 2.0 ** -34 * top, 0)
    return out, bound
