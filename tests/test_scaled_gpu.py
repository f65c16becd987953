"""Operators with run-time scales on the GPU: quantize_rows_i8 bit for bit against the
rational definition, linear_scaled_i8 against the product in 64 bits."""
import numpy as np
import pytest

from guard import Guarded

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ip():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_30846_gb300 as ip
    ip.load()
    return ip


def quant_ref(x):
    """q and scale of the definition: float64 holds 127 x exactly, and a quotient that is
    no half integer is further from one than its rounding."""
    v = x.double().cpu().numpy()
    top = np.abs(v).max(-1, keepdims=True)
    ok = np.isfinite(top) & (top > 0)
    with np.errstate(all="ignore"):
        q = np.where(ok, np.rint(127.0 * v / np.where(ok, top, 1.0)), 0.0)
        s = np.where(np.isfinite(top), (top / 127.0).astype(np.float32), np.float32("nan"))
    return q.astype(np.int8), s[..., 0].astype(np.float32)


def same_quant(ip, x, **kw):
    q, s = ip.quantize_rows_i8(x, **kw)
    wq, ws = quant_ref(x)
    np.testing.assert_array_equal(s.cpu().numpy(), ws)
    np.testing.assert_array_equal(q.cpu().numpy(), wq)
    return q, s


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 7), (3, 8), (5, 33), (2, 1000), (9, 1024), (4, 1025),
                                    (300, 129), (7, 4096), (3, 4100), (2, 8192), (2, 8193), (1, 32768)])
def test_quantize_matches_definition(ip, dtype, rows, d):
    g = torch.Generator(device="cuda").manual_seed(rows * 40000 + d)
    x = (torch.randn(rows, d, generator=g, device="cuda") * 3).to(DT[dtype])
    same_quant(ip, x)


@pytest.mark.parametrize("dtype", list(DT))
def test_quantize_ties_and_neighbours(ip, dtype):
    # x = (2 n + 1) c with amax = 254 c is a tie for every n; the neighbours of the
    # ties in the type's grid are not
    dt = DT[dtype]
    rows = []
    for c in (1.0, 3.0, 5.0, 7.0, 0.37, 1.1e-3):
        c = float(torch.tensor(c, dtype=dt))
        odd = torch.arange(1, 254, 2, dtype=torch.float64) * c
        t = odd.to(dt)
        bits = t.view(torch.int32 if dt == torch.float32 else torch.int16)
        near = torch.cat([t, (bits + 1).view(dt), (bits - 1).view(dt)])
        top = torch.tensor([254.0 * c], dtype=torch.float64).to(dt)
        keep = near[near.double() <= top.double()]
        row = torch.cat([top, keep, -keep])
        rows.append(torch.cat([row, torch.zeros(800 - row.numel(), dtype=dt)]))
    same_quant(ip, torch.stack(rows).cuda())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_quantize_every_pair_of_significands(ip, dtype):
    # a row for every significand of amax, with every significand below it in nine binades:
    # all quotients that the 16-bit types can have in the rounding's reach, ties among them
    dt, bits = DT[dtype], 10 if dtype == "f16" else 7
    sig = torch.arange(1 << bits, 2 << bits, device="cuda", dtype=torch.float64) * 2.0 ** -bits
    vals = torch.cat([sig * 2.0 ** -j for j in range(9)])
    for top in sig.split(128):
        x = torch.where(vals[None] <= top[:, None], vals[None], torch.zeros((), device="cuda", dtype=torch.float64))
        x = torch.cat([top[:, None], x, -x], 1).to(dt)
        q, s = ip.quantize_rows_i8(x)
        want = (127.0 * x.double() / top[:, None]).round()     # exact enough: 53 bits, ties representable
        assert torch.equal(q.double(), want)
        assert torch.equal(s.double(), (top / 127.0).float().double())


@pytest.mark.parametrize("scale", [1e-45, 1e-42, 1e-38, 3e-37, 1e-20, 1e20, 1e36, 3e38])
def test_quantize_extreme_ranges(ip, scale):
    g = torch.Generator(device="cuda").manual_seed(3)
    x = (torch.rand(6, 517, generator=g, device="cuda", dtype=torch.float64) * 2 - 1) * scale
    x = x.float()
    x[0] = 0
    x[1, 1:] = 0
    same_quant(ip, x)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
def test_quantize_not_finite(ip, dtype, bad):
    x = torch.randn(4, 300, device="cuda").to(DT[dtype])
    x[1, 299] = float(bad)
    q, s = same_quant(ip, x)
    assert torch.isnan(s[1]) and not q[1].any()
    w = torch.randint(-127, 128, (16, 304), dtype=torch.int8, device="cuda")[:, :300]
    y = ip.linear_scaled_i8(q, s, w, torch.ones(16, device="cuda"), dtype=torch.float32)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[[0, 2, 3]]).all()


def test_quantize_strides_and_untouched_bytes(ip):
    base = torch.randn(3, 5, 700, device="cuda").to(torch.bfloat16)
    for x in (base[..., 3:260], base[..., 8:520], base[:, 2], base[1:2, :, :9]):
        same_quant(ip, x)
    g = Guarded((5, 320), torch.int8)
    before = g.view.clone()
    x = base[0, :, :301]
    q, s = same_quant(ip, x, q=g.view[:, :301])
    assert torch.equal(g.view[:, 301:], before[:, 301:])
    g.check()


def product_ref(x, sx, w, sw, bias, swish):
    """The definition in float64: |sums| < 2^53 are exact."""
    y = x.double() @ w.double().t() * sx.double()[:, None] * sw.double()
    if bias is not None:
        y = y + bias.double()
    return y * torch.sigmoid(y) if swish else y


def product_bound(x, sx, w, sw, bias, swish, dt):
    """Bound of the kernel's error, from its roundings: the sum to f32, the product of the
    scales, one fused multiply-add: z is off by at most (2 |s sx sw| + |z|) 2^-24 (1 + 2^-20);
    the activation's slope is at most 1.1, its own arithmetic is charged 2^-20 relative
    (2^-18 with the fast exponential of the 16-bit outputs and |z| 2^-22 more for
    the rounding of its argument); then half a step of the output's type."""
    s = (x.double() @ w.double().t()).abs() * sx.double()[:, None] * sw.double()
    z = product_ref(x, sx, w, sw, bias, False).abs()
    e = (2 * s + z) * 2.0 ** -24 * 1.001
    y = product_ref(x, sx, w, sw, bias, swish).abs()
    if swish:
        e = 1.1 * e + y * (2.0 ** -20 if dt == torch.float32 else 2.0 ** -18 + z * 2.0 ** -22)
    tiny = torch.finfo(dt).smallest_normal
    return e + (y + e) * torch.finfo(dt).eps / 2 + tiny * torch.finfo(dt).eps


def check_product(ip, M, K, N, dt, swish=False, bias=True, seed=0, lo=-127, hi=127, out=None):
    g = torch.Generator(device="cuda").manual_seed(seed + M + 7 * K + 13 * N)
    ri = lambda r, c: torch.randint(lo, hi + 1, (r, -(-c // 16) * 16), generator=g, device="cuda",
                                    dtype=torch.int8)[:, :c]
    x, w = ri(M, K), ri(N, K)
    sx = torch.rand(M, generator=g, device="cuda") * 0.02 / K ** 0.5
    sw = torch.rand(N, generator=g, device="cuda") * 0.05
    b = torch.randn(N, generator=g, device="cuda") if bias else None
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    y = ip.linear_scaled_i8(x, sx, w, sw, b, act=ip.ACT_SWISH if swish else ip.ACT_NONE, dtype=dt,
                            workspace=ws, out=out)
    assert ip.status(ws) == 0
    err = (y.double() - product_ref(x, sx, w, sw, b, swish)).abs()
    assert (err <= product_bound(x, sx, w, sw, b, swish, dt)).all(), float(err.max())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 16, 5), (2, 100, 33), (3, 1024, 64), (4, 1000, 1000),
                                   (5, 17, 640), (8, 4096, 1024), (7, 2049, 5000), (1, 1024, 20000),
                                   (9, 64, 32), (9, 1, 1), (33, 100, 77), (127, 1024, 256), (128, 63, 128),
                                   (129, 65, 129), (200, 1025, 300), (333, 1000, 777), (257, 4096, 96),
                                   (1000, 128, 5000), (2500, 520, 2100), (3000, 2100, 1030),
                                   (17, 4096, 1024), (100, 8192, 70), (129, 3000, 33), (12, 32768, 40)])
def test_product(ip, dtype, M, K, N):
    check_product(ip, M, K, N, DT[dtype])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("M,K,N", [(1, 1024, 4096), (6, 300, 50), (125, 1024, 4096), (700, 200, 3000)])
def test_product_swish(ip, dtype, M, K, N):
    check_product(ip, M, K, N, DT[dtype], swish=True, bias=M != 6)


@pytest.mark.parametrize("M,N", [(3, 40), (40, 64), (140, 300), (64, 16384), (2600, 2048)])
@pytest.mark.parametrize("K", [1024, 1040, 2048, 5000])
def test_sums_are_exact_at_the_extremes(ip, M, N, K):
    # every product has the largest magnitude: the partial sums reach 2^24 in each
    # segment, and the two halves of K cancel up to a few units
    ld = -(-K // 16) * 16
    x = torch.full((M, ld), -128, dtype=torch.int8, device="cuda")[:, :K]
    w = torch.full((N, ld), -128, dtype=torch.int8, device="cuda")[:, :K]
    x[1::2, K // 2:] = 127
    w[::3, ::2] = 127
    w[::5, -1] = 1
    one = lambda n: torch.ones(n, device="cuda")
    y = ip.linear_scaled_i8(x, one(M), w, one(N), dtype=torch.float32)
    want = (x.double() @ w.double().t()).float()     # exact in 64 bits, one rounding to f32
    assert torch.equal(y, want)


def test_rows_and_columns_outside_are_left(ip):
    for M, K, N, ldy in ((5, 40, 30, 37), (140, 70, 45, 64), (300, 1100, 200, 208)):
        for dt in (torch.float32, torch.bfloat16):
            g = Guarded((M, ldy), dt)
            before = g.view.clone()
            check_product(ip, M, K, N, dt, out=g.view[:, :N])
            assert torch.equal(g.view[:, N:].contiguous().view(torch.uint8),
                               before[:, N:].contiguous().view(torch.uint8))
            g.check()


def test_other_stream_and_graph(ip):
    x = torch.randn(2, 70, 256, device="cuda").to(torch.float16)
    wq, sw = ip.quantize_rows_i8(torch.randn(300, 256, device="cuda"))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")

    def step(stream=None):
        q, s = ip.quantize_rows_i8(x, stream=stream)
        return ip.linear_scaled_i8(q, s, wq, sw, dtype=torch.float16, workspace=ws, stream=stream)
    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = step(side)
    side.synchronize()
    assert torch.equal(got, want) and got.shape == (2, 70, 300)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step())
    assert ip.status(ws) == 0


def test_empty(ip):
    q, s = ip.quantize_rows_i8(torch.zeros(0, 64, device="cuda"))
    assert q.shape == (0, 64) and s.shape == (0,)
    w = torch.zeros(8, 64, dtype=torch.int8, device="cuda")
    assert ip.linear_scaled_i8(q, s, w, torch.ones(8, device="cuda")).shape == (0, 8)


@pytest.mark.parametrize("M", [5, 90, 3000])
def test_rows_without_a_scale_and_far_activations(ip, M):
    # rows of zeros, rows that were not finite, and a swish far out on both sides, in each form
    x = torch.randn(M, 640, device="cuda").to(torch.bfloat16)
    x[1] = 0
    x[3, 5] = float("inf")
    w, sw = ip.quantize_rows_i8(torch.randn(1500, 640, device="cuda") * 9)
    b = torch.linspace(-120, 120, 1500, device="cuda")
    q, s = ip.quantize_rows_i8(x)
    for dt in DT.values():
        y = ip.linear_scaled_i8(q, s, w, sw, b, act=ip.ACT_SWISH, dtype=dt)
        assert torch.isnan(y[3]).all()
        keep = [i for i in range(M) if i != 3]
        err = (y[keep].double() - product_ref(q[keep], s[keep], w, sw, b, True)).abs()
        # below exp(-87) the exponential itself is a subnormal number: 2^-149 off, times |z|
        assert (err <= product_bound(q[keep], s[keep], w, sw, b, True, dt) + 2.0 ** -140).all()
        z = b.double()
        want = z * torch.sigmoid(z)
        tol = want.abs() * (2.0 ** -17 + z.abs() * 2.0 ** -21 + torch.finfo(dt).eps / 2) + 2.0 ** -140 + \
            torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
        assert ((y[1].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("M,K,N", [(40, 1024, 1500), (100, 4096, 100), (1000, 1024, 1037), (900, 2100, 1033),
                                   (2000, 1024, 4097), (1001, 2100, 4090)])
@pytest.mark.parametrize("shift,ld", [(0, 0), (1, 3), (4, 8), (2, 2)])
def test_output_rows_of_any_alignment(ip, dtype, M, K, N, shift, ld):
    # the same bits whatever the rows' alignment, and nothing beside them
    g = torch.Generator(device="cuda").manual_seed(M)
    q, s = ip.quantize_rows_i8(torch.randn(M, K, generator=g, device="cuda"))
    w, sw = ip.quantize_rows_i8(torch.randn(N, K, generator=g, device="cuda"))
    b = torch.randn(N, generator=g, device="cuda")
    wide = torch.empty(M, (N + 31) // 32 * 32, dtype=DT[dtype], device="cuda")
    base = torch.full((M, N + shift + ld), 7.0, dtype=DT[dtype], device="cuda")
    for act in (ip.ACT_NONE, ip.ACT_SWISH):
        want = ip.linear_scaled_i8(q, s, w, sw, b, act=act, out=wide[:, :N])
        ip.linear_scaled_i8(q, s, w, sw, b, act=act, out=base[:, shift:shift + N])
        assert torch.equal(base[:, shift:shift + N], want)
        assert (base[:, :shift] == 7).all() and (base[:, shift + N:] == 7).all()
    z = (q[:9].double() @ w.double().t()) * s[:9, None].double() * sw.double() + b.double()
    mag = (q[:9].double() @ w.double().t()).abs() * s[:9, None].double() * sw.double() + b.double().abs()
    got = ip.linear_scaled_i8(q, s, w, sw, b, out=base[:, shift:shift + N])[:9].double()
    fin = torch.finfo(DT[dtype])
    # sx sw, the sum to f32 and the multiply-add round once each (2^-24), then the output
    tol = mag * 4 * 2.0 ** -24 + z.abs() * fin.eps / 2 * 1.01 + fin.smallest_normal * fin.eps
    assert ((got - z).abs() <= tol).all()


def test_offsets_past_31_bits(ip):
    M, N, K = 36000, 65536, 48
    x = torch.randint(-127, 128, (M, K), dtype=torch.int8, device="cuda")
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda")
    one = lambda n: torch.ones(n, device="cuda")
    y = ip.linear_scaled_i8(x, one(M), w, one(N), dtype=torch.float16)
    assert y.numel() > 2 ** 31
    for r in (slice(0, 3), slice(32760, 32776), slice(M - 3, M)):
        assert torch.equal(y[r].double(), (x[r].double() @ w.double().t()).half().double())
    base = torch.zeros(40, 1 << 26, dtype=torch.int8, device="cuda")     # rows 64 MB apart
    base[:, :K] = x[:40]
    assert torch.equal(ip.linear_scaled_i8(base[:, :K], one(40), w[:300], one(300), dtype=torch.float32),
                       ip.linear_scaled_i8(x[:40], one(40), w[:300], one(300), dtype=torch.float32))
    xf = torch.randn(40, 1 << 26, device="cuda", dtype=torch.float16)
    q, s = ip.quantize_rows_i8(xf[:, -K:])
    q2, s2 = ip.quantize_rows_i8(xf[:, -K:].contiguous())
    assert torch.equal(q, q2) and torch.equal(s, s2)


def test_seeded_sweep(ip):
    rng = np.random.default_rng(77)
    for i in range(60):
        M, K, N = (int(round(np.exp(rng.uniform(0, np.log(t))))) for t in (5000, 9000, 6000))
        if M * K * N > 4e10:
            K = max(1, int(4e10 / M / N))
        check_product(ip, M, K, N, list(DT.values())[i % 3], swish=bool(rng.random() < 0.5),
                      bias=bool(rng.random() < 0.5), seed=i, lo=-128)


def test_refusals(ip):
    x = torch.zeros(4, 64, dtype=torch.int8, device="cuda")
    w, s4, s8 = torch.zeros(8, 64, dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda"), torch.ones(8, device="cuda")
    ok = dict(x=x, sx=s4, w=w, sw=s8)
    ip.linear_scaled_i8(**ok)
    odd = torch.zeros(4, 65, dtype=torch.int8, device="cuda")
    for err, over in ((ValueError, dict(sx=s8)), (ValueError, dict(sw=s4)), (TypeError, dict(sx=s4.half())),
                      (TypeError, dict(x=x.float())), (TypeError, dict(w=w.cpu())), (ValueError, dict(w=w[:, :48])),
                      (ValueError, dict(bias=s4)), (TypeError, dict(dtype=torch.float64)),
                      (ip.IpError, dict(x=odd[:, :64])), (ip.IpError, dict(x=odd[:, 1:], w=w)),
                      (ip.IpError, dict(act=7)), (ValueError, dict(x=x.t())),
                      (ValueError, dict(x=x[:1].expand(4, 64))),
                      (ValueError, dict(out=torch.zeros(4, 9, device="cuda"))),
                      (ValueError, dict(workspace=torch.zeros(512, dtype=torch.uint8, device="cuda")[::2])),
                      (ip.IpError, dict(workspace=torch.zeros(128, dtype=torch.uint8, device="cuda")))):
        with pytest.raises(err):
            ip.linear_scaled_i8(**dict(ok, **over))
    for err, t in ((TypeError, x), (TypeError, torch.zeros(3, 4)), (ValueError, torch.zeros(4, 6, device="cuda").t()),
                   (ValueError, torch.zeros(2, 3, 4, device="cuda").transpose(0, 1)),
                   (ValueError, torch.zeros(3, 0, device="cuda")),
                   (ip.IpError, torch.zeros(1, 40000, device="cuda"))):
        with pytest.raises(err):
            ip.quantize_rows_i8(t)
