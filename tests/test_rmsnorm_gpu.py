"""The root-mean-square norm with quantised rows on the GPU against its definition in float64: codes bit
for bit, scales to the rounding of their sum of squares."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import fp4_ref as ref

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ip():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_30846_gb300 as ip
    ip.load()
    return ip


def tolerance(d):
    # a thread adds 32 squares in turn (d / 256 where a row is longer than 8192), then a tree of up to 12 levels:
    # each addition of positive numbers is relative 2^-24, each square too; the root halves it;
    # then the mean, eps, the root, the reciprocal and two more products
    return ((max(32, d / 256) + 13) / 2 + 7) * 2.0 ** -24


def i8_codes(z):
    top = z.abs().amax(1, keepdim=True)
    ok = torch.isfinite(top) & (top > 0)
    return torch.where(ok, (127.0 * z / torch.where(ok, top, 1.0)).round(), 0.0)


def check(ip, x, g, res=None, eps=1e-5, **kw):
    """Both forms against float64; returns what they gave."""
    d, lead = x.shape[-1], x.shape[:-1]
    h = x if res is None else (x.double() + res.double()).to(x.dtype)
    flat = h.reshape(-1, d)
    z = (flat.double() * g.double()).float().double()
    fin = torch.isfinite(z.abs().amax(1))
    rstd = (flat.double().square().mean(1) + eps).rsqrt()
    q, s, t = ip.rmsnorm_i8(x, g, res, eps=eps, **kw)
    assert q.shape == x.shape and s.shape == lead and (t is None) == (res is None)
    if res is not None:
        assert torch.equal(t.float().nan_to_num(7), h.float().nan_to_num(7)) and t.dtype == x.dtype
    assert torch.equal(q.reshape(-1, d).double(), i8_codes(z))
    want = torch.where(fin, torch.where(z.abs().amax(1) > 0, z.abs().amax(1) * rstd / 127, 0.0), float("nan"))
    near = lambda a, b: bool((torch.isnan(a) == torch.isnan(b)).all() and
                             ((a - b).abs().nan_to_num(0) <= tolerance(d) * b.abs().nan_to_num(0) + 2.0 ** -149).all())
    assert near(s.reshape(-1).double(), want)
    q4, b4, s4, t4 = ip.rmsnorm_fp4(x, g, res, eps=eps, **kw)
    c, sb, r = ref.quantize(z)
    wq, wb = ref.bytes_of(c, sb)
    free = ref.untouched(b4, flat.shape[0])
    assert torch.equal(q4.reshape(wq.shape), wq) and torch.equal(b4[~free], wb[~free])
    assert near(s4.reshape(-1).double(), torch.where(r > 0, r * rstd, r))
    if res is not None:
        assert torch.equal(t4.float().nan_to_num(7), h.float().nan_to_num(7))
    return q, s, t, q4, b4, s4


def draw(rows, d, dtype, seed, res=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *n: torch.randn(*n, generator=g, device="cuda")
    gain = 1 + 20 * (torch.rand(d, generator=g, device="cuda") < 0.02)
    return ((rnd(rows, d) * gain).to(dtype), (1 + 0.3 * rnd(d)).to(dtype), rnd(rows, d).to(dtype) if res else None)


@pytest.mark.parametrize("res", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 7), (3, 8), (5, 33), (130, 64), (2, 1000), (9, 1024), (4, 1025),
                                    (301, 129), (7, 4096), (3, 4100), (2, 8192), (2, 8193), (1, 32768)])
def test_matches_definition(ip, dtype, rows, d, res):
    x, g, r = draw(rows, d, DT[dtype], rows * 40000 + d, res)
    check(ip, x, g, r)


def test_many_rows(ip):
    x, g, r = draw(12001, 257, torch.bfloat16, 5)
    check(ip, x, g, r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-42, 1e-38, 1e-25, 1e-12, 1e12, 1e18, 1e25, 3e38])
@pytest.mark.parametrize("eps", [0.0, 1e-5, 1e20])
def test_extreme_ranges(ip, dtype, scale, eps):
    for d in (300, 2000, 9000):
        x, g, _ = draw(5, d, torch.float32, d, False)
        x = (x / x.abs().amax(1, keepdim=True) * scale).to(DT[dtype])
        g = (g / g.abs().amax()).to(DT[dtype])
        x[1] = 0
        x[2, 1:] = 0
        if scale == 1e-42:
            g[:] = 1
        if eps == 0.0 and scale == 3e38:
            continue                # 1 / rms below the normal numbers
        check(ip, x, g, eps=eps)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,weight", [(1e17, 1e20), (1e30, 1e7), (1e20, 1e-38), (1e-12, 1e-30), (1e-20, 1e-20), (1e-12, 1e30),
                                          (1e-30, 1e20)])
def test_extreme_weights(ip, dtype, scale, weight):
    # the scale itself is well inside f32's range, its factors are not
    for d in (300, 2000, 9000):
        x, g, _ = draw(5, d, torch.float32, d, False)
        check(ip, (x / x.abs().amax() * scale).to(DT[dtype]), (g / g.abs().amax() * weight).to(DT[dtype]), eps=0.0)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
def test_not_finite(ip, dtype, bad):
    for d in (300, 2000, 9000):
        x, g, r = draw(5, d, DT[dtype], 1)
        x[1, d - 1] = float(bad)
        r[3, 0] = float(bad)
        q, s = check(ip, x, g, r)[:2]
        assert torch.isnan(s).tolist() == [False, True, False, True, False]


def test_overflowing_sum_and_product(ip):
    x = torch.full((2, 40), 60000.0, device="cuda").half()
    x[1] = 1
    one = torch.ones(40, device="cuda").half()
    s, t = ip.rmsnorm_i8(x, one, x.clone())[1:]
    assert torch.isinf(t[0]).all() and torch.isnan(s[0]) and torch.isfinite(s[1])
    x = torch.full((2, 40), 2e38, device="cuda")
    x[1] = 1
    s = ip.rmsnorm_i8(x, 4 * torch.ones(40, device="cuda"))[1]
    assert torch.isnan(s[0]) and torch.isfinite(s[1])


@pytest.mark.parametrize("d", [96, 100, 3000, 9001])
def test_sum_in_place(ip, d):
    x, g, r = draw(37, d, torch.bfloat16, d)
    want = [t.clone() for t in ip.rmsnorm_i8(x, g, r)]
    for where in ("x", "res"):
        a, b = x.clone(), r.clone()
        got = ip.rmsnorm_i8(a, g, b, out=a if where == "x" else b)
        assert all(torch.equal(u, v) for u, v in zip(got, want))
        a, b = x.clone(), r.clone()
        got = ip.rmsnorm_fp4(a, g, b, out=a if where == "x" else b)
        assert torch.equal(got[3], want[2])


def test_strides(ip):
    base, g, _ = draw(12, 1400, torch.float16, 9)
    x, r = base[:, 3:260], base[:, 700:957]
    wide = torch.full((12, 300), 5.0, device="cuda").half()
    q = torch.full((12, 290), 9, dtype=torch.int8, device="cuda")
    got = check(ip, x, g[:257].contiguous(), r)
    ip.rmsnorm_i8(x, g[:257].contiguous(), r, out=wide[:, 7:264], q=q[:, 1:258])
    assert torch.equal(wide[:, 7:264], got[2]) and torch.equal(q[:, 1:258], got[0])
    assert (wide[:, :7] == 5).all() and (wide[:, 264:] == 5).all() and (q[:, 0] == 9).all() and (q[:, 258:] == 9).all()
    x3 = base.view(3, 4, 1400)[..., 8:520]
    check(ip, x3, g[:512].contiguous(), x3)
    assert ip.rmsnorm_i8(x[:0], g[:257].contiguous())[0].shape == (0, 257)


def test_a_stream_of_its_own_and_a_graph(ip):
    x, g, r = draw(64, 1024, torch.bfloat16, 11)
    want = ip.rmsnorm_fp4(x, g, r)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = ip.rmsnorm_fp4(x, g, r, stream=side)
    side.synchronize()
    mine = ~ref.untouched(want[1], 64)           # bytes of rows behind the last are not written
    assert all(torch.equal(a, b) for a, b in zip((*got, got[1][mine]), (*want, want[1][mine])) if a.dim() != 3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, b, s, t = ip.rmsnorm_fp4(x, g, r)
        y = ip.dequantize_fp4(q, b, s)
    x.copy_(x.flip(0))
    r.copy_(r.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s, want[2].flip(0)) and torch.equal(t, want[3].flip(0))
    assert torch.equal(y, ip.dequantize_fp4(*want[:3]).flip(0))


def test_refusals(ip):
    x, g, r = draw(4, 64, torch.float16, 1)
    for f in (ip.rmsnorm_i8, ip.rmsnorm_fp4):
        for err, args, kw in ((TypeError, (x.cpu(), g), {}), (TypeError, (x.double(), g.double()), {}), (TypeError, (x, g.float()), {}),
                              (ValueError, (x, g[:63]), {}), (ValueError, (x, g, r[:3]), {}), (TypeError, (x, g, r.float()), {}),
                              (ValueError, (x, g), dict(out=r)), (ValueError, (x, g, r), dict(out=r[:, :63])),
                              (ip.IpError, (x, g), dict(eps=-1.0)), (ip.IpError, (x, g), dict(eps=float("nan"))),
                              (ValueError, (x.t(), g[:4]), {}), (ValueError, (x, g, r), dict(scale=torch.zeros(3, device="cuda"))),
                              (ValueError, (x, torch.ones(128, device="cuda").half()[::2]), {})):
            with pytest.raises(err):
                f(*args, **kw)
