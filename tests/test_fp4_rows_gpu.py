"""4-bit rows on the GPU: quantize_fp4 bit for bit against the definition in float64, the values
of rows, and what the calls refuse."""
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


def same(ip, x, **kw):
    d = x.shape[-1]
    flat = x.reshape(-1, d)
    rows = flat.shape[0]
    blocks = torch.full(ip.fp4_block_shape(rows, d), 0xA5, dtype=torch.uint8, device="cuda")
    q, b, s = ip.quantize_fp4(x, blocks=blocks, **kw)
    wq, wb = ref.bytes_of(*ref.quantize(flat)[:2])
    ws = ref.quantize(flat)[2]
    assert b is blocks
    gs = s.reshape(-1).double()
    assert torch.equal(torch.isnan(gs), torch.isnan(ws)) and torch.equal(gs.nan_to_num(7), ws.nan_to_num(7))
    free = ref.untouched(blocks, rows)
    assert torch.equal(blocks[~free], wb[~free]) and (blocks[free] == 0xA5).all()
    assert torch.equal(q.reshape(rows, -1), wq)
    return q, b, s


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 15), (3, 8), (5, 33), (130, 64), (2, 1000), (9, 1024), (4, 1025),
                                    (300, 129), (7, 4096), (3, 4100), (2, 8192), (2, 8193), (1, 32768)])
def test_matches_definition(ip, dtype, rows, d):
    g = torch.Generator(device="cuda").manual_seed(rows * 40000 + d)
    x = torch.randn(rows, d, generator=g, device="cuda") * (1 + 30 * (torch.rand(d, generator=g, device="cuda") < 0.02))
    same(ip, x.to(DT[dtype]))


@pytest.mark.parametrize("dtype", list(DT))
def test_ties_and_neighbours(ip, dtype):
    # blocks whose largest element is 6 s: every midpoint of the codes times s, and its neighbours in the
    # type's grid; blocks whose largest element is a midpoint between two scales times 6, and its neighbours
    dt = DT[dtype]
    it = torch.int32 if dt == torch.float32 else torch.int16
    up = lambda t, k: (t.view(it) + k).view(dt)
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    s = torch.tensor(ref.E4M3[8:], dtype=torch.float64)
    rows = []
    for k in (-1, 0, 1):
        t = up((mids[None] * s[:, None]).to(dt), k)
        rows.append(torch.cat([(6 * s)[:, None].to(dt), t, -t, torch.zeros(len(s), 1, dtype=dt)], 1).flatten())
    half = (s[:-1] + s[1:]) / 2 * 6
    for k in (-1, 0, 1):
        t = up(half.to(dt), k)
        rows.append(torch.cat([t[:, None], t[:, None] / 3, torch.zeros(len(t), 14, dtype=dt)], 1).flatten())
    rows = [torch.cat([torch.full((16,), 2688.0, dtype=dt), r]) for r in rows]
    for r in rows:
        same(ip, r[None].cuda())
        if dt != torch.float16:
            same(ip, r[None].cuda() * 2.0 ** -20)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_every_significand_as_row_maximum(ip, dtype):
    dt, bits = DT[dtype], 10 if dtype == "f16" else 7
    sig = torch.arange(1 << bits, 2 << bits, device="cuda", dtype=torch.float64) * 2.0 ** -bits
    vals = torch.cat([sig[:: max(1, len(sig) // 128)] * 2.0 ** -j for j in range(8)])
    x = torch.where(vals[None] <= sig[:, None], vals[None], 0.0)
    same(ip, torch.cat([sig[:, None], x, -x], 1).to(dt))


@pytest.mark.parametrize("scale", [1e-45, 1e-42, 3e-36, 1e-35, 1e-20, 1e20, 1e36, 3e38])
def test_extreme_ranges(ip, scale):
    g = torch.Generator(device="cuda").manual_seed(3)
    x = ((torch.rand(6, 517, generator=g, device="cuda", dtype=torch.float64) * 2 - 1) * scale).float()
    x[0] = 0
    x[1, 1:] = 0
    x[2, 16:] *= 2.0 ** -40
    x[3, 16:] *= 2.0 ** -17
    same(ip, x)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
def test_not_finite(ip, dtype, bad):
    x = torch.randn(4, 300, device="cuda").to(DT[dtype])
    x[1, 299] = float(bad)
    q, b, s = same(ip, x)
    assert torch.isnan(s[1]) and not q[1].any()
    y = ip.dequantize_fp4(q, b, s, 300)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[[0, 2, 3]]).all()


def test_strides_and_untouched_bytes(ip):
    base = torch.randn(3, 5, 700, device="cuda").to(torch.bfloat16)
    for x in (base[..., 3:260], base[..., 8:520], base[:, 2], base[1:2, :, :9], base[..., :33]):
        same(ip, x)
    g = Guarded((5, 320), torch.uint8)
    before = g.view.clone()
    same(ip, base[0, :, :301], q=g.view[:, :151])
    assert torch.equal(g.view[:, 151:], before[:, 151:])
    g.check()
    assert ip.quantize_fp4(base[:0])[0].shape == (0, 5, 350)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 17), (130, 100), (200, 1024), (5, 32768)])
def test_values(ip, dtype, rows, d):
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(rows, d, generator=g, device="cuda")
    q, b, s = ip.quantize_fp4(x)
    s = s * torch.rand(rows, generator=g, device="cuda")
    want = ref.values(q.reshape(rows, -1), b, s, d)
    got = ip.dequantize_fp4(q, b, s, d, dtype=DT[dtype])
    # f32 values are one rounding; the others the rounding of that one
    assert torch.equal(got, want.float().to(DT[dtype]))
    out = torch.full((rows, d + 3), 7.0, dtype=DT[dtype], device="cuda")
    ip.dequantize_fp4(q, b, s, d, out=out[:, 1:d + 1])
    assert torch.equal(out[:, 1:d + 1], got) and (out[:, [0, -1, -2]] == 7).all()
    q8, s8 = ip.quantize_rows_i8(x)
    got = ip.dequantize_i8(q8, s8, dtype=DT[dtype])
    assert torch.equal(got, (q8.double() * s8.double()[:, None]).float().to(DT[dtype]))
    ip.dequantize_i8(q8, s8, out=out[:, 2:d + 2])
    assert torch.equal(out[:, 2:d + 2], got) and (out[:, -1] == 7).all()


def test_every_byte_of_codes_and_scales(ip):
    q = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(254, 1)                # 512 elements a row
    sb = torch.cat([torch.arange(127), torch.arange(128, 255)]).to(torch.uint8).cuda()     # any scale but NaN
    _, blocks = ref.bytes_of(torch.zeros(254, 2, dtype=torch.uint8, device="cuda"), sb[:, None].repeat(1, 32))
    s = torch.full((254,), 3.0, device="cuda")
    assert torch.equal(ip.dequantize_fp4(q, blocks, s, dtype=torch.float32).double(), ref.values(q, blocks, s, 512))


def test_refusals(ip):
    x = torch.randn(4, 64, device="cuda")
    q, b, s = ip.quantize_fp4(x)
    for err, call in ((TypeError, lambda: ip.quantize_fp4(x.cpu())), (TypeError, lambda: ip.quantize_fp4(x.double())),
                      (ValueError, lambda: ip.quantize_fp4(x, q=q[:, 1:])), (TypeError, lambda: ip.quantize_fp4(x, q=q.char())),
                      (ValueError, lambda: ip.quantize_fp4(x, blocks=b[:, :, :511])),
                      (ValueError, lambda: ip.quantize_fp4(x, scale=s[:3])), (ValueError, lambda: ip.quantize_fp4(x.t())),
                      (ip.IpError, lambda: ip.quantize_fp4(x, q=torch.empty(4, 40, dtype=torch.uint8, device="cuda")[:, :32])),
                      (ValueError, lambda: ip.dequantize_fp4(q, b, s, 61)), (ValueError, lambda: ip.dequantize_fp4(q, b, s, 65)),
                      (TypeError, lambda: ip.dequantize_fp4(q, b, s, dtype=torch.int32)),
                      (ValueError, lambda: ip.dequantize_fp4(q, b, s[:3])), (TypeError, lambda: ip.dequantize_i8(q, s)),
                      (ValueError, lambda: ip.dequantize_i8(q.view(torch.int8), s, out=torch.empty(4, 31, device="cuda")))):
        with pytest.raises(err):
            call()
