"""More rows than a grid has groups of threads for (2^20 CTAs): each group then takes several rows in turn, with
the same buffers.  What it gives for them all is what it gives for a part of them at a time."""
import pytest

from test_rmsnorm_gpu import ip  # noqa: F401 - a fixture

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

CTAS = 1 << 20


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def parts(rows):
    """Slices of less than the grid's own, on multiples of 128 rows (a group of block scales)."""
    step = rows // 3 // 128 * 128
    return slice(0, step), slice(step, 2 * step), slice(2 * step, rows)


def scales_of(b, rows):
    """Block scales as [rows, bytes] in the rows' order."""
    t, s = b.shape[:2]
    return b.view(t, s, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(t * 128, 4 * s)[:rows]


# four rows a CTA; then a row a CTA of four warps.  An odd length: rows that are not on 16 bytes.
@pytest.mark.parametrize("rows,d", [(4 * CTAS + 5, 17), (4 * CTAS + 131, 16), (CTAS + 3, 1025), (CTAS + 129, 1032)])
def test_norm_and_rows(ip, rows, d):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(d)
    rnd = lambda *n: torch.randn(*n, generator=g, device="cuda", dtype=torch.float32).bfloat16()
    x, r, w = rnd(rows, d), rnd(rows, d), rnd(d)
    q, s, t = ip.rmsnorm_i8(x, w, r)
    for p in parts(rows):
        assert all(torch.equal(a[p], b) for a, b in zip((q, s, t), ip.rmsnorm_i8(x[p], w, r[p])))
    del q, s, t
    for call in (lambda p: ip.rmsnorm_fp4(x[p], w, r[p]), lambda p: ip.quantize_fp4(x[p])):
        q, b, s = call(slice(None))[:3]
        for p in parts(rows):
            u, v, z = call(p)[:3]
            assert torch.equal(q[p], u) and torch.equal(s[p], z)
            assert torch.equal(scales_of(b, rows)[p], scales_of(v, len(u)))
        del q, b, s, u, v, z


# 16 elements a thread: whole ones on 16 bytes, and rows of one
@pytest.mark.parametrize("d", [16, 1])
def test_values(ip, d):  # noqa: F811
    rows = 256 * CTAS + 300
    g = torch.Generator(device="cuda").manual_seed(d)
    s = torch.rand(rows, generator=g, device="cuda")
    q = torch.randint(-128, 128, (rows, d), generator=g, device="cuda", dtype=torch.int8)
    y = ip.dequantize_i8(q, s)
    for p in parts(rows):
        assert torch.equal(y[p], ip.dequantize_i8(q[p], s[p]))
    del y, q
    q = torch.randint(0, 256, (rows, 16), generator=g, device="cuda", dtype=torch.uint8)[:, :(d + 1) // 2]
    b = torch.randint(0, 127, ip.fp4_block_shape(rows, d), generator=g, device="cuda", dtype=torch.uint8)
    y = ip.dequantize_fp4(q, b, s, d)
    for p in parts(rows):
        assert torch.equal(y[p], ip.dequantize_fp4(q[p], b[p.start // 128:-(-p.stop // 128)], s[p], d))
