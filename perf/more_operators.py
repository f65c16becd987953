"""Performance cases of a decoder's operators around its products: the root-mean-square norm with
the residual's addition and rows quantised in the same pass (to int8, or to microscaled 4-bit
floating point), the product in that 4-bit format, and the log probabilities at the end of a step.

Shapes are those of the library's encoder (d = 1024, feed-forward 4096, 125 frames for a 10 s
utterance, 32 x 375 = 12000 frames for its batch, a vocabulary of 1024 tokens and the blank) and of
an autoregressive decoder behind it.  A case is a plain dict:

  norm      x [M, D] (+ residual [M, D]) -> rmsnorm_i8 or rmsnorm_fp4; the sum and the rows' values
  linear    x [M, K] -> quantize_fp4 -> linear_fp4 with weights [N, K]
  logprobs  logits [M, V], tokens [M] -> log probability, entropy, the `top` best tokens

4-bit rows: a code is the e2m1 number of a nibble (sign, then 0 .5 1 1.5 2 3 4 6), low nibble first; each 16
consecutive elements share an e4m3 scale s, a row an f32 scale r; an element is code s r.  The e4m3 bytes
lie in blocks of 512 for 128 rows x 64 elements: [rows / 128, K / 64, row mod 32, (row mod 128) / 32, 4].
"""
import math
import random

import torch

own = False      # True: the library's operators; False: plain torch

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # the norm in front of a block's products for the one token of one user: latency
        dict(name="norm token 1x1024 i8", kind="norm", M=1, D=1024, to="i8", res=True, dtype="bf16"),
        # rows that divide by nothing, the first norm (nothing to add yet), 4-bit rows
        dict(name="norm odd 333x1000 fp4", kind="norm", M=333, D=1000, to="fp4", res=False, dtype="f16"),
        # the encoder batch's frames with their residual
        dict(name="norm batch 12000x1024 i8", kind="norm", M=12000, D=1024, to="i8", res=True, dtype="bf16"),
        # a decoder's feed-forward product for the one token of one user: latency
        dict(name="linear token 1x1024x4096", kind="linear", M=1, K=1024, N=4096, dtype="bf16",
             swish=True, bias=True),
        # the way back for one 10 s utterance
        dict(name="linear utterance 125x4096x1024", kind="linear", M=125, K=4096, N=1024, dtype="f16",
             swish=False, bias=False),
        # sizes that divide by nothing, 32-bit in and out
        dict(name="linear odd 333x1000x777", kind="linear", M=333, K=1000, N=777, dtype="f32",
             swish=False, bias=True),
        # the encoder batch, both feed-forward products
        dict(name="linear batch 12000x1024x4096", kind="linear", M=12000, K=1024, N=4096,
             dtype="bf16", swish=True, bias=True),
        dict(name="linear batch 12000x4096x1024", kind="linear", M=12000, K=4096, N=1024,
             dtype="f16", swish=False, bias=True),
        # one token's logits over a large vocabulary, with the best alternatives: latency
        dict(name="logprobs token 1x65536", kind="logprobs", M=1, V=65536, top=20, dtype="f32"),
        # a batch's tokens over a large vocabulary
        dict(name="logprobs tokens 64x65536", kind="logprobs", M=64, V=65536, top=8, dtype="bf16"),
        # the frames of four utterances of up to two minutes over the small vocabulary, one best token each
        dict(name="logprobs frames 1500x1025", kind="logprobs", M=1500, V=1025, top=1, dtype="f16"),
        # scoring the encoder batch's frames, no alternatives asked for
        dict(name="logprobs batch 12000x1025", kind="logprobs", M=12000, V=1025, top=0, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "linear", "logprobs"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    if kind == "norm":
        D = _log(rng, 16, 8192)
        return dict(kind=kind, M=_log(rng, 1, max(1, min(12000, 12000 * 512 // D))), D=D,
                    to=rng.choice(["i8", "fp4"]), res=rng.random() < 0.6, dtype=dtype)
    if kind == "linear":
        K, N = _log(rng, 48, 4096), _log(rng, 48, 4096)
        # within the products and the bytes of the listed batch cases
        most = min(12000, 12000 * 1024 * 4096 // (K * N), 12000 * 5120 * 2 // ((K + N) * BYTES[dtype]))
        return dict(kind=kind, M=_log(rng, 1, most), K=K, N=N, dtype=dtype,
                    swish=rng.random() < 0.5, bias=rng.random() < 0.7)
    V = _log(rng, 32, 131072)
    return dict(kind=kind, M=_log(rng, 1, max(1, min(12000, 12000 * 512 // V))), V=V,
                top=rng.choice([0, 1, 5, 20, 32]), dtype=dtype)


def work(case):
    e, M = BYTES[case["dtype"]], case["M"]
    if case["kind"] == "norm":
        n = M * case["D"]
        # x (and the residual) in, the sum, the quantised rows and their values out
        code = 1.0 if case["to"] == "i8" else 9 / 16
        return {"bytes": n * (e * (3 if case["res"] else 1) + code + 4) + case["D"] * e + 4 * M, "flops": 8.0 * n}
    if case["kind"] == "linear":
        K, N = case["K"], case["N"]
        return {"bytes": M * K * e + N * K * 9 / 16 + 4 * N * (2 if case["bias"] else 1) + M * N * e,
                "flops": 2.0 * M * K * N}
    return {"bytes": M * (case["V"] * e + 4 + 8 + 8 * case["top"]), "flops": 6.0 * M * case["V"]}


# ------------------------------------------------------------------ inputs

def _pow2(e):
    """2^e (float64) for integers e: the bits of its exponent (torch.ldexp goes through a power in 32 bits)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _round_e4m3(y):
    """The e4m3 numbers nearest to 0 <= y <= 448 (float64), ties to even."""
    u = _pow2(torch.frexp(y)[1].clamp(min=-5) - 4)            # the step at y; the least normal number is 2^-6
    return torch.round(y / u) * u


def _round_e2m1(y):
    """The e2m1 numbers nearest to y (float64), ties to even."""
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0).double()).double()
    return torch.copysign((torch.round(a / step) * step).clamp(max=6.0), y)


def _quant_fp4(x):
    """Codes [M, B, 16], block scales [M, B] and row scales [M] (float64) of rows [M, K] (B = ceil(K / 16))."""
    v = torch.nn.functional.pad(x.double(), (0, -x.shape[1] % 16)).unflatten(1, (-1, 16))
    top = v.abs().amax(-1)
    f, e = torch.frexp(top.amax(-1))                          # amax = f 2^e, f in [0.5, 1)
    e = torch.where(f <= 0.65625, e - 12, e - 11).clamp(min=-126)
    r = _pow2(e)
    s = _round_e4m3(top / (6.0 * r[:, None]))
    d = (s * r[:, None]).unsqueeze(-1)
    return torch.where(d > 0, _round_e2m1(v / torch.where(d > 0, d, 1.0)), 0.0), s, r


def _pack_fp4(c, s):
    """Bytes of codes and scales in the library's layout: uint8 [M, 16 k], uint8 [M / 128, K / 64, 512]."""
    a = c.abs()
    n = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    n = (n | (torch.signbit(c).to(torch.uint8) << 3)).flatten(1).unflatten(1, (-1, 2))
    q = n[..., 0] | (n[..., 1] << 4)
    q = torch.nn.functional.pad(q, (0, -q.shape[1] % 16))
    M, B = s.shape
    m, e = torch.frexp(s)                                     # normal: 1.mmm 2^(e - 1), exponent field e + 6
    byte = torch.where(s < 2.0 ** -6, s * 512, (e + 6) * 8 + (16 * m - 8)).to(torch.uint8)
    byte = torch.nn.functional.pad(byte, (0, -B % 4, 0, -M % 128))
    b = byte.unflatten(0, (-1, 4, 32)).unflatten(3, (-1, 4)).permute(0, 3, 2, 1, 4)
    return q, b.reshape(b.shape[0], b.shape[1], 512).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    rand = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")
    dt, M = DTYPES[case["dtype"]], case["M"]
    if case["kind"] == "norm":
        D = case["D"]
        # a residual stream with a few strong channels, and a block's output to add to it
        gain = 1.0 + 15.0 * (rand(D) < 0.01)
        return {"case": case, "x": (rnd(M, D) * (gain if not case["res"] else 0.5)).to(dt),
                "res": (2.0 * rnd(M, D) * gain).to(dt) if case["res"] else None,
                "g": (1.0 + 0.2 * rnd(D)).to(dt)}
    if case["kind"] == "linear":
        K, N = case["K"], case["N"]
        # normalised activations with a few strong channels
        x = (rnd(M, K) * (1.0 + 7.0 * (rand(K) < 0.01))).to(dt)
        c, s, r = _quant_fp4(rnd(N, K) * (0.5 + rand(N, 1)) / math.sqrt(K))
        w, wb = _pack_fp4(c, s)
        return {"case": case, "x": x, "w": w[:, :-(-K // 2)], "wb": wb, "sw": r.float(),
                "bias": rnd(N) if case["bias"] else None, "ws": None}
    V = case["V"]
    # logits as a head gives them: a few tokens stand out, some tokens are ruled out
    x = 2.0 * rnd(M, V) + 8.0 * (rand(M, V) < 4.0 / V)
    x = torch.where(rand(V) < 0.01, -math.inf, x)
    x[:, 0] = 1.0
    return {"case": case, "x": x.to(dt), "ws": None,
            "tokens": torch.randint(0, V, (M,), generator=gen, device="cuda", dtype=torch.int32)}


# ------------------------------------------------------------------ plain torch

def _plain_norm(st):
    h = st["x"].float() if st["res"] is None else (st["x"].float() + st["res"].float()).to(st["x"].dtype).float()
    z = h * st["g"].float()
    rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    if st["case"]["to"] == "i8":
        top = z.abs().amax(1, keepdim=True)
        q = (127.0 * z.double() / torch.where(top > 0, top, 1.0)).round().float()    # next to half integers 32 bits lose
        values = q * (top * rstd / 127.0)
    else:
        c, s, r = _quant_fp4(z)
        values = (c * s.unsqueeze(-1)).flatten(1)[:, :z.shape[1]].float() * (r[:, None].float() * rstd)
    return {"values": values} if st["res"] is None else {"sum": h.to(st["x"].dtype), "values": values}


def _weights(st):
    """f32 [N, K] without the row scales, from the packed bytes."""
    w, wb, K = st["w"], st["wb"], st["case"]["K"]
    n = torch.stack([w & 15, w >> 4], -1).flatten(1)[:, :K]
    m = (n & 7).float()
    c = torch.where(m < 4, m / 2, torch.where(m < 6, m - 2, 2 * m - 8)) * (1.0 - 2.0 * (n >> 3).float())
    b = wb.unflatten(2, (32, 4, 4)).permute(0, 3, 2, 1, 4).flatten(0, 2).flatten(1)[:w.shape[0]]
    e, f = (b >> 3).float(), (b & 7).float()
    s = torch.where(e > 0, torch.exp2(e - 7) * (1 + f / 8), f / 512)
    return c * s.repeat_interleave(16, 1)[:, :K]


def _plain_linear(st):
    c, s, r = _quant_fp4(st["x"])
    xq = (c * s.unsqueeze(-1)).flatten(1)[:, :st["case"]["K"]].float()
    y = (xq @ _weights(st).t()) * (r[:, None].float() * st["sw"])
    if st["bias"] is not None:
        y = y + st["bias"]
    if st["case"]["swish"]:
        y = y / (1.0 + torch.exp(-y))
    return y.to(st["x"].dtype)


def _plain_logprobs(st):
    x, top = st["x"].float(), st["case"]["top"]
    a = x - x.amax(1, keepdim=True)
    e = torch.exp(a)
    s = e.sum(1)
    ls = torch.log(s)
    ent = ls - (e * torch.where(e > 0, a, 0.0)).sum(1) / s
    out = {"logprob": a.gather(1, st["tokens"].long()[:, None])[:, 0] - ls, "entropy": ent}
    if top:
        # stable: among equal logits the lowest index first
        v, i = torch.sort(x, dim=1, descending=True, stable=True)
        out["top_logprob"] = v[:, :top] - x.amax(1, keepdim=True) - ls[:, None]
        out["top_token"] = i[:, :top].to(torch.int32)
    return out


# ------------------------------------------------------------------ the library's operators

def _workspace(st, size):
    # a user's program keeps its workspace between calls
    if st["ws"] is None:
        st["ws"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    return st["ws"]


def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"norm": _plain_norm, "linear": _plain_linear, "logprobs": _plain_logprobs}[kind](st)
    import paper_2609_30846_gb300 as ip
    if kind == "norm":
        if case["to"] == "i8":
            q, scale, total = ip.rmsnorm_i8(st["x"], st["g"], st["res"], eps=EPS)
            values = ip.dequantize_i8(q, scale, dtype=torch.float32)
        else:
            q, blocks, scale, total = ip.rmsnorm_fp4(st["x"], st["g"], st["res"], eps=EPS)
            values = ip.dequantize_fp4(q, blocks, scale, case["D"], dtype=torch.float32)
        return {"values": values} if st["res"] is None else {"sum": total, "values": values}
    if kind == "linear":
        q, blocks, scale = ip.quantize_fp4(st["x"])
        return ip.linear_fp4(q, blocks, scale, st["w"], st["wb"], st["sw"], st["bias"],
                             act=ip.ACT_SWISH if case["swish"] else ip.ACT_NONE,
                             dtype=st["x"].dtype, workspace=_workspace(st, 256))
    size = 0 if st["ws"] is not None else ip.token_logprobs_workspace_bytes(case["M"], case["V"], case["top"])
    lp, ent, top_lp, top_tok = ip.token_logprobs(st["x"], st["tokens"], top=case["top"],
                                                 workspace=_workspace(st, size))
    if not case["top"]:
        return {"logprob": lp, "entropy": ent}
    return {"logprob": lp, "entropy": ent, "top_logprob": top_lp, "top_token": top_tok}


# ------------------------------------------------------------------ 64-bit values

_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
_E4M3 = [m / 512 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1]


def _nearest(y, grid):
    """The number of the ascending grid nearest to y >= 0, the one of even index between two."""
    g = torch.tensor(grid, dtype=torch.float64, device="cuda")
    i = torch.searchsorted(g, y.contiguous()).clamp(max=len(grid) - 1)       # g[i - 1] < y <= g[i]
    lo = (i - 1).clamp(min=0)
    below, above = y - g[lo], g[i] - y
    return g[torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, i)]


def _fp4_values(x):
    """Rows [M, K] (float64) rounded to 4-bit rows, as (values over the row scale, row scales)."""
    K = x.shape[1]
    top = x.abs().max(1).values
    # the least power of two r with top <= 2688 r
    k = torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 2688)).to(torch.int32)
    two = torch.full_like(top, 2.0)
    k = torch.where(top <= 2688 * two.pow(k - 1), k - 1, k)
    k = torch.where(top > 2688 * two.pow(k), k + 1, k)
    r = (k.clamp(min=-126).long() + 1023 << 52).view(torch.float64)
    out = torch.zeros_like(x)
    for at in range(0, K, 16):
        part = x[:, at:at + 16] / r[:, None]
        s = _nearest(part.abs().max(1).values / 6, _E4M3)[:, None]
        c = _nearest((part / torch.where(s == 0, 1.0, s)).abs(), _E2M1) * part.sign()
        out[:, at:at + 16] = torch.where(s == 0, 0.0, c * s)
    return out, r


def exact(case, seed):
    st = prepare(case, seed)
    x = st["x"].to(torch.float64)
    if case["kind"] == "norm":
        h = x if st["res"] is None else (x + st["res"].to(torch.float64)).to(st["x"].dtype).to(torch.float64)
        z = (h * st["g"].to(torch.float64)).to(torch.float32).to(torch.float64)   # the product is defined in 32 bits
        inv = (h.square().sum(1) / case["D"] + EPS) ** -0.5
        if case["to"] == "i8":
            top = z.abs().max(1).values
            k = torch.floor(2 * 127 * z.abs() / top[:, None])             # in half steps, rounded down
            n = torch.div(k, 2, rounding_mode="floor")
            tie = 2 * 127 * z.abs() == (2 * n + 1) * top[:, None]
            n = torch.where(tie, n + n % 2, torch.where(k % 2 == 1, n + 1, n))
            values = n * z.sign() * (top * inv / 127)[:, None]
        else:
            v, r = _fp4_values(z)
            values = v * (r * inv)[:, None]
        return {"values": values} if st["res"] is None else {"sum": h, "values": values}
    if case["kind"] == "linear":
        N, K = case["N"], case["K"]
        n, k = torch.arange(N, device="cuda")[:, None], torch.arange(K, device="cuda")[None]
        nib = (st["w"][n, k // 2].to(torch.int64) >> (4 * (k % 2))) & 15
        byte = st["wb"][n // 128, k // 64, n % 32 * 16 + n % 128 // 32 * 4 + k // 16 % 4].to(torch.int64)
        table = lambda v: torch.tensor(v, dtype=torch.float64, device="cuda")
        w = table(_E2M1 + [-v for v in _E2M1])[nib] * table(_E4M3 + [math.nan])[byte]
        v, r = _fp4_values(x)
        y = torch.einsum("mk,nk->mn", v, w) * r[:, None] * st["sw"].to(torch.float64)[None]
        if case["bias"]:
            y = y + st["bias"].to(torch.float64)
        return y * torch.sigmoid(y) if case["swish"] else y
    lse = torch.logsumexp(x, 1)
    p = torch.softmax(x, 1)
    out = {"logprob": x[torch.arange(case["M"], device="cuda"), st["tokens"].long()] - lse,
           "entropy": -torch.special.xlogy(p, p).sum(1)}
    if case["top"]:
        # one 64-bit key a token: its logit's order, then its index from behind
        b = (st["x"].float() + 0.0).view(torch.int32).long()
        b = torch.where(b < 0, -(b & 0x7FFFFFFF), b)
        i = torch.topk(b * (1 << 20) + (case["V"] - 1 - torch.arange(case["V"], device="cuda")), case["top"], 1).indices
        out["top_logprob"], out["top_token"] = x.gather(1, i) - lse[:, None], i.to(torch.int32)
    return out
