"""The product of 4-bit rows on the GPU against float64."""
import pytest

from guard import Guarded

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


def rows(n, k, seed, scales=True):
    """Random 4-bit rows made without the library: (q, blocks, scale), q with rows of a multiple of 16 bytes, junk behind."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.randint(0, 16, (n, k), generator=g, device="cuda", dtype=torch.uint8)
    B = -(-k // 16)
    sb = torch.randint(8, 90, (n, B), generator=g, device="cuda", dtype=torch.uint8) if scales else torch.full(
        (n, B), 0x38, dtype=torch.uint8, device="cuda")
    q, blocks = ref.bytes_of(c, sb)
    blocks = torch.where(ref.untouched(blocks, n), torch.full_like(blocks, 255), blocks)     # rows behind the last: NaN
    pad = torch.full((n, -q.shape[1] % 16 + 16), 0x77, dtype=torch.uint8, device="cuda")
    scale = 0.5 + torch.rand(n, generator=g, device="cuda") if scales else torch.ones(n, device="cuda")
    return torch.cat([q, pad], 1)[:, :q.shape[1]], blocks, scale


SIZES = [(1, 1, 1), (1, 16, 8), (1, 64, 64), (3, 40, 17), (128, 64, 64), (128, 256, 64), (7, 300, 100), (128, 512, 128), (130, 1000, 777),
         (1, 1024, 4096), (2, 1025, 130), (4, 4000, 257), (5, 2080, 1000), (8, 4096, 1024), (8, 33, 129), (9, 1024, 512), (64, 4096, 1024), (300, 1100, 200), (9, 32768, 70), (129, 5000, 65), (1000, 4000, 300), (125, 4096, 1024), (333, 1000, 777), (200, 2000, 9728), (2000, 100, 1024), (1500, 1024, 4096),
         (2049, 333, 4097), (40, 32768, 33), (5000, 576, 3000), (1000, 2048, 5001)]


@pytest.mark.parametrize("M,K,N", SIZES)
def test_sums_of_codes_are_exact(ip, M, K, N):
    # scales of 1: products are multiples of 1/4 and sums stay below 2^22
    x, w = rows(M, K, M + K, False), rows(N, K, N + K, False)
    want = ref.values(*x, K) @ ref.values(*w, K).t()
    y = ip.linear_fp4(*x, *w, dtype=torch.float32)
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("swish,bias", [(False, False), (True, True)])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_matches_float64(ip, M, K, N, swish, bias, dtype):
    x, w = rows(M, K, M + K), rows(N, K, N + K)
    vx, vw = ref.values(*x, K), ref.values(*w, K)
    b = torch.randn(N, device="cuda") * 100 if bias else None
    out = Guarded((M, N), DT[dtype])
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    y = ip.linear_fp4(*x, *w, b, act=ip.ACT_SWISH if swish else ip.ACT_NONE, out=out.view, workspace=ws)
    out.check()
    assert ip.status(ws) == 0
    z = vx @ vw.t() + (b.double() if bias else 0)
    # sums of K / 16 scaled blocks in f32, each addition off by at most 2^-23 of the magnitudes so far; the scales' product, the
    # fma, f32 again; swish changes by at most 1.1 per unit and is off by a few 2^-22 of |z|
    off = ((K / 16 + 8) * 2.0 ** -23) * (vx.abs() @ vw.abs().t()) + 2.0 ** -23 * z.abs()
    want = z * torch.sigmoid(z) if swish else z
    if swish:
        off = 1.1 * off + 2.0 ** -20 * z.abs()
    fin = torch.finfo(DT[dtype])
    off = off * (1 + fin.eps) + fin.eps / 2 * want.abs() + fin.smallest_normal * fin.eps
    keep = want.abs() < 0.9 * fin.max
    assert ((y.double() - want).abs() <= off)[keep].all()


def test_a_scale_at_a_time(ip):
    # one block of x and of w at a time has another scale: each scale meets its own block
    M, K, N = 260, 320, 300
    x, w = rows(M, K, 1, False), rows(N, K, 2, False)
    for b in range(K // 16):
        for m, n in ((0, 0), (31, 32), (33, 63), (64, 64), (100, 127), (127, 128), (128, 200), (259, 299)):
            xb, wb = x[1].clone(), w[1].clone()
            xb[m // 128, b // 4, 16 * (m % 32) + 4 * (m % 128 // 32) + b % 4] = 0x38 + 16       # 4
            wb[n // 128, b // 4, 16 * (n % 32) + 4 * (n % 128 // 32) + b % 4] = 0x38 - 12       # 0.375
            y = ip.linear_fp4(x[0], xb, x[2], w[0], wb, w[2], dtype=torch.float32)
            assert torch.equal(y.double(), ref.values(x[0], xb, x[2], K) @ ref.values(w[0], wb, w[2], K).t())


def test_quantised_rows(ip):
    x, w = torch.randn(300, 1000, device="cuda").bfloat16(), torch.randn(500, 1000, device="cuda")
    a, b = ip.quantize_fp4(x), ip.quantize_fp4(w)
    y = ip.linear_fp4(*a, *b, dtype=torch.float32).double()
    want = ref.values(*a, 1000) @ ref.values(*b, 1000).t()
    assert ((y - want).abs() <= (1000 / 16 + 8) * 2.0 ** -23 * (ref.values(*a, 1000).abs() @ ref.values(*b, 1000).abs().t())).all()
    full = x.double() @ w.double().t()
    assert ((y - full).norm() / full.norm()) < 0.2      # two operands of 4 bits, about 0.1 each


def test_rows_that_are_not_finite(ip):
    x = torch.randn(5, 200, device="cuda")
    x[1, 3] = float("nan")
    x[3, 199] = float("inf")
    y = ip.linear_fp4(*ip.quantize_fp4(x), *ip.quantize_fp4(torch.randn(40, 200, device="cuda")))
    assert torch.isnan(y).all(1).tolist() == [False, True, False, True, False] and torch.isfinite(y[[0, 2, 4]]).all()


@pytest.mark.parametrize("dtype", list(DT))
def test_a_channel_or_a_bias_that_is_not_finite(ip, dtype):
    for M, K, N in ((3, 64, 100), (300, 256, 512), (2000, 128, 2050)):
        x, w = rows(M, K, 1), rows(N, K, 2)
        bias = torch.randn(N, device="cuda")
        want = ip.linear_fp4(*x, *w, bias, act=ip.ACT_SWISH, dtype=DT[dtype])
        w[2][5], bias[N - 2], bias[17], bias[18] = float("nan"), float("nan"), float("inf"), -float("inf")
        y = ip.linear_fp4(*x, *w, bias, act=ip.ACT_SWISH, dtype=DT[dtype])
        own = torch.tensor([5, 17, 18, N - 2], device="cuda")
        assert torch.isnan(y[:, [5, N - 2]]).all() and (y[:, 17] == float("inf")).all() and (y[:, 18] == 0).all()
        assert torch.equal(y.index_fill(1, own, 0), want.index_fill(1, own, 0))


@pytest.mark.parametrize("dtype", list(DT))
def test_output_rows_of_any_alignment(ip, dtype):
    for M, K, N in ((70, 100, 95), (300, 200, 2000), (3000, 128, 3001)):
        x, w = rows(M, K, 5), rows(N, K, 6)
        want = ip.linear_fp4(*x, *w, dtype=DT[dtype])
        for shift in (0, 1, 2, 4, 7):
            base = torch.full((M, N + 21), 3.0, dtype=DT[dtype], device="cuda")
            ip.linear_fp4(*x, *w, out=base[:, shift:shift + N])
            assert torch.equal(base[:, shift:shift + N], want)
            assert (base[:, :shift] == 3).all() and (base[:, shift + N:] == 3).all()


def test_leading_axes_no_rows_and_strides(ip):
    x = torch.randn(3, 50, 128, device="cuda")
    w = ip.quantize_fp4(torch.randn(96, 128, device="cuda"))
    q, b, s = ip.quantize_fp4(x)
    y = ip.linear_fp4(q, b, s, *w)
    assert y.shape == (3, 50, 96) and torch.equal(y.view(150, 96), ip.linear_fp4(q.view(150, 64), b, s.view(150), *w))
    e = ip.quantize_fp4(x[:0])
    assert ip.linear_fp4(*e, *w).shape == (0, 50, 96)
    wide = torch.zeros(150, 208, dtype=torch.uint8, device="cuda")
    wide[:, 16:80] = q.view(150, 64)
    assert torch.equal(ip.linear_fp4(wide[:, 16:80], b, s.view(150), *w), y.view(150, 96))
    # the first 128 channels of more
    w = ip.quantize_fp4(torch.randn(300, 128, device="cuda"))
    y = ip.linear_fp4(q, b, s, *w)
    assert torch.equal(ip.linear_fp4(q, b, s, w[0][:128], w[1][:1], w[2][:128]), y[..., :128])


def test_streams_and_graphs(ip):
    x, w = rows(500, 1024, 1), rows(2048, 1024, 2)
    want = ip.linear_fp4(*x, *w)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    ys = [ip.linear_fp4(*x, *w, stream=s) for s in (a, b, a, b)]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in ys)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ip.linear_fp4(*x, *w, workspace=ws)
        z = ip.linear_fp4(*ip.quantize_fp4(y), *ip.quantize_fp4(y[:40]), workspace=ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(z, ip.linear_fp4(*ip.quantize_fp4(want), *ip.quantize_fp4(want[:40])))


def test_refusals(ip):
    x, w = ip.quantize_fp4(torch.randn(4, 64, device="cuda")), ip.quantize_fp4(torch.randn(8, 64, device="cuda"))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    ok = dict(zip(("x", "x_blocks", "sx", "w", "w_blocks", "sw"), (*x, *w)))
    ip.linear_fp4(**ok)
    for err, over in ((TypeError, dict(x=x[0].char())), (TypeError, dict(w=w[0].cpu())), (ValueError, dict(x_blocks=x[1][:, :, :256])),
                      (ValueError, dict(w=w[0][:, :16])), (ValueError, dict(sw=w[2][:7])), (TypeError, dict(sx=x[2].double())),
                      (ValueError, dict(bias=torch.zeros(7, device="cuda"))), (ip.IpError, dict(act=2)),
                      (TypeError, dict(dtype=torch.float64)), (ValueError, dict(out=torch.zeros(4, 7, device="cuda"))),
                      (ip.IpError, dict(workspace=ws[:128])), (ip.IpError, dict(workspace=torch.zeros(512, dtype=torch.uint8, device="cuda")[16:])),
                      (ip.IpError, dict(x=torch.zeros(4, 40, dtype=torch.uint8, device="cuda")[:, :32])),
                      (ValueError, dict(w_blocks=torch.zeros(2, 1, 512, dtype=torch.uint8, device="cuda")))):
        with pytest.raises(err):
            ip.linear_fp4(**dict(ok, **over))
