"""Refusals of the norm, the 4-bit rows and their product, the values of rows and the log probabilities,
without a GPU: every case fails validation before any pointer is used."""
import ctypes

import pytest

import paper_2609_30846_gb300 as ip

P = ctypes.c_void_p
A = 1 << 20
FAKE, WS = P(A), P(2 * A)
NULL, SHAPE, ALIGN, PARAM, WORKSPACE = -1, -2, -3, -7, -8
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return ip.load()


def refusals(fn, order, base, none, cases):
    run = lambda **o: fn(*[dict(base, **o)[n] for n in order])
    assert run(rows=0, **{n: None for n in none}) == 0           # no rows: no pointer is touched
    for over, code in cases:
        assert run(**over) == code, over


ROWS = ((dict(dtype=3), PARAM), (dict(dtype=-1), PARAM), (dict(rows=-1), SHAPE), (dict(rows=(1 << 40) + 1), SHAPE), (dict(d=0), SHAPE),
        (dict(d=32769), SHAPE))
FP4 = ((dict(ldq=49), SHAPE), (dict(ldq=1 << 41), SHAPE), (dict(q=None), NULL), (dict(blocks=None), NULL), (dict(scale=None), NULL),
       (dict(q=P(A + 8)), ALIGN), (dict(ldq=56), ALIGN), (dict(blocks=P(A + 4)), ALIGN), (dict(scale=P(A + 2)), ALIGN))


def test_block_bytes(lib):
    f = lib.ip_fp4_block_bytes
    assert [f(0, 64), f(1, 1), f(128, 64), f(129, 64), f(128, 65), f(1, 32768)] == [0, 512, 512, 1024, 1024, 512 * 512]
    assert f(1, 0) == f(1, 32769) == f(-1, 64) == f((1 << 40) + 1, 64) == 0
    assert f(1 << 40, 32768) == (1 << 33) * 512 * 512
    assert ip.fp4_block_shape(130, 100) == (2, 2, 512)


def test_quantize_fp4(lib):
    refusals(lib.ip_quantize_fp4, ("x", "dtype", "rows", "d", "ldx", "q", "ldq", "blocks", "scale", "stream"),
             dict(x=FAKE, dtype=2, rows=4, d=100, ldx=100, q=FAKE, ldq=64, blocks=FAKE, scale=FAKE, stream=None),
             ("x", "q", "blocks", "scale"),
             ROWS + FP4 + ((dict(ldx=99), SHAPE), (dict(x=None), NULL), (dict(x=P(A + 1)), ALIGN), (dict(dtype=0, x=P(A + 2)), ALIGN)))


NORM = dict(x=FAKE, ldx=100, res=FAKE, ldr=100, w=FAKE, eps=1e-5, dtype=1, rows=4, d=100, sum=FAKE, lds=100, q=FAKE, scale=FAKE, stream=None)
NORM_CASES = ROWS + (
    (dict(eps=-1e-9), PARAM), (dict(eps=NAN), PARAM), (dict(eps=INF), PARAM), (dict(eps=1e30), PARAM), (dict(ldx=99), SHAPE),
    (dict(ldr=99), SHAPE), (dict(lds=99), SHAPE), (dict(ldx=(1 << 40) + 1), SHAPE), (dict(x=None), NULL), (dict(w=None), NULL),
    (dict(sum=None), NULL), (dict(x=P(A + 1)), ALIGN), (dict(w=P(A + 1)), ALIGN), (dict(res=P(A + 1)), ALIGN), (dict(sum=P(A + 1)), ALIGN),
    (dict(dtype=0, w=P(A + 2)), ALIGN))


def test_rmsnorm_i8(lib):
    refusals(lib.ip_rmsnorm_i8, ("x", "ldx", "res", "ldr", "w", "eps", "dtype", "rows", "d", "sum", "lds", "q", "ldq", "scale", "stream"),
             dict(NORM, ldq=100), ("x", "res", "w", "sum", "q", "scale"),
             NORM_CASES + ((dict(ldq=99), SHAPE), (dict(q=None), NULL), (dict(scale=None), NULL), (dict(scale=P(A + 2)), ALIGN)))


def test_rmsnorm_fp4(lib):
    refusals(lib.ip_rmsnorm_fp4,
             ("x", "ldx", "res", "ldr", "w", "eps", "dtype", "rows", "d", "sum", "lds", "q", "ldq", "blocks", "scale", "stream"),
             dict(NORM, ldq=64, blocks=FAKE), ("x", "res", "w", "sum", "q", "blocks", "scale"), NORM_CASES + FP4)


def test_values(lib):
    Y = ((dict(ldy=99), SHAPE), (dict(y=None), NULL), (dict(y=P(A + 1)), ALIGN), (dict(dtype=0, y=P(A + 2)), ALIGN))
    refusals(lib.ip_dequantize_i8, ("q", "ldq", "scale", "rows", "d", "y", "ldy", "dtype", "stream"),
             dict(q=FAKE, ldq=100, scale=FAKE, rows=4, d=100, y=FAKE, ldy=100, dtype=2, stream=None), ("q", "scale", "y"),
             ROWS + Y + ((dict(ldq=99), SHAPE), (dict(q=None), NULL), (dict(scale=None), NULL), (dict(scale=P(A + 1)), ALIGN)))
    refusals(lib.ip_dequantize_fp4, ("q", "ldq", "blocks", "scale", "rows", "d", "y", "ldy", "dtype", "stream"),
             dict(q=FAKE, ldq=64, blocks=FAKE, scale=FAKE, rows=4, d=100, y=FAKE, ldy=100, dtype=2, stream=None),
             ("q", "blocks", "scale", "y"), ROWS + Y + FP4)


def test_linear_fp4(lib):
    refusals(lib.ip_linear_fp4, ("x", "ldx", "xb", "sx", "w", "ldw", "wb", "sw", "bias", "act", "rows", "K", "N", "y", "ldy", "dtype", "ws",
                                 "wsb", "stream"),
             dict(x=FAKE, ldx=64, xb=FAKE, sx=FAKE, w=FAKE, ldw=64, wb=FAKE, sw=FAKE, bias=None, act=0, rows=4, K=100, N=50, y=FAKE, ldy=50,
                  dtype=2, ws=WS, wsb=256, stream=None), ("x", "xb", "sx", "w", "wb", "sw", "y", "ws"),
             ((dict(dtype=3), PARAM), (dict(act=2), PARAM), (dict(act=-1), PARAM), (dict(rows=-1), SHAPE), (dict(rows=(1 << 27) + 1), SHAPE),
              (dict(K=0), SHAPE), (dict(K=32769, ldx=1 << 15, ldw=1 << 15), SHAPE), (dict(N=0), SHAPE), (dict(N=65537, ldy=65537), SHAPE),
              (dict(ldx=48), SHAPE), (dict(ldw=48), SHAPE), (dict(ldy=49), SHAPE), (dict(ldx=1 << 40), SHAPE), (dict(ldy=(1 << 31) + 1), SHAPE),
              (dict(x=None), NULL), (dict(xb=None), NULL), (dict(sx=None), NULL), (dict(w=None), NULL), (dict(wb=None), NULL),
              (dict(sw=None), NULL), (dict(y=None), NULL), (dict(ws=None), NULL), (dict(x=P(A + 8)), ALIGN), (dict(w=P(A + 4)), ALIGN),
              (dict(ldx=56), ALIGN), (dict(ldw=72), ALIGN), (dict(xb=P(A + 8)), ALIGN), (dict(wb=P(A + 1)), ALIGN), (dict(sx=P(A + 2)), ALIGN),
              (dict(sw=P(A + 2)), ALIGN), (dict(bias=P(A + 2)), ALIGN), (dict(y=P(A + 1)), ALIGN), (dict(dtype=0, y=P(A + 2)), ALIGN),
              (dict(ws=P(2 * A + 128)), ALIGN), (dict(wsb=255), WORKSPACE)))


def test_token_logprobs(lib):
    size = lib.ip_token_logprobs_workspace_bytes
    assert size(4, 1000, 5) == 256 and size(0, 1000, 0) == 256 and size(1, 130000, 32) == 256
    assert size(3, 1 << 20, 20) > size(3, 1 << 20, 0) > 256
    for bad in ((-1, 10, 0), (4, 0, 0), (4, (1 << 20) + 1, 0), (4, 100, 33), (4, 100, -1), (4, 5, 6), ((1 << 27) + 1, 10, 0)):
        assert size(*bad) == 0, bad
    with pytest.raises(ip.IpError):
        ip.token_logprobs_workspace_bytes(4, 5, 6)
    refusals(lib.ip_token_logprobs, ("x", "dtype", "rows", "V", "ld", "tok", "wide", "scale", "top", "lp", "ent", "tlp", "ttok", "ws", "wsb", "stream"),
             dict(x=FAKE, dtype=1, rows=4, V=1000, ld=1000, tok=FAKE, wide=0, scale=1.0, top=5, lp=FAKE, ent=FAKE, tlp=FAKE, ttok=FAKE, ws=WS,
                  wsb=256, stream=None), ("x", "tok", "lp", "ent", "tlp", "ttok", "ws"),
             ((dict(dtype=3), PARAM), (dict(scale=0.0), PARAM), (dict(scale=-1.0), PARAM), (dict(scale=NAN), PARAM), (dict(scale=INF), PARAM),
              (dict(wide=2), PARAM), (dict(rows=-1), SHAPE), (dict(rows=(1 << 27) + 1), SHAPE), (dict(V=0), SHAPE),
              (dict(V=(1 << 20) + 1, ld=1 << 21), SHAPE), (dict(ld=999), SHAPE), (dict(ld=(1 << 40) + 1), SHAPE), (dict(top=33), SHAPE),
              (dict(top=-1), SHAPE), (dict(V=4, top=5), SHAPE), (dict(x=None), NULL), (dict(ent=None), NULL), (dict(ws=None), NULL),
              (dict(lp=None), NULL), (dict(tlp=None), NULL), (dict(ttok=None), NULL), (dict(x=P(A + 1)), ALIGN), (dict(dtype=0, x=P(A + 2)), ALIGN),
              (dict(tok=P(A + 2)), ALIGN), (dict(wide=1, tok=P(A + 4)), ALIGN), (dict(lp=P(A + 2)), ALIGN), (dict(ent=P(A + 2)), ALIGN),
              (dict(tlp=P(A + 2)), ALIGN), (dict(ttok=P(A + 2)), ALIGN), (dict(ws=P(2 * A + 64)), ALIGN), (dict(wsb=255), WORKSPACE),
              (dict(V=1 << 20, ld=1 << 20, wsb=1000), WORKSPACE)))


def test_sizes_past_32_bits(lib):
    # what an int does not hold is refused, not wrapped into a size that is offered
    for big in ((1 << 32) + 64, (1 << 32) + 1, -(1 << 32) + 64):
        assert lib.ip_quantize_fp4(FAKE, 2, 4, big, 1 << 39, FAKE, 1 << 39, FAKE, FAKE, None) == SHAPE
        assert lib.ip_rmsnorm_i8(FAKE, 1 << 39, None, 0, FAKE, 1e-5, 1, 4, big, None, 0, FAKE, 1 << 39, FAKE, None) == SHAPE
        assert lib.ip_dequantize_i8(FAKE, 1 << 39, FAKE, 4, big, FAKE, 1 << 39, 2, None) == SHAPE
        assert lib.ip_token_logprobs(FAKE, 1, 4, big, 1 << 39, None, 0, 1.0, 0, None, FAKE, None, None, WS, 256, None) == SHAPE
        assert lib.ip_token_logprobs(FAKE, 1, 4, 100, 100, None, 0, 1.0, big, None, FAKE, FAKE, FAKE, WS, 256, None) == SHAPE
        for K, N in ((big, 50), (100, big)):
            assert lib.ip_linear_fp4(FAKE, 1 << 38, FAKE, FAKE, FAKE, 1 << 38, FAKE, FAKE, None, 0, 4, K, N, FAKE, 1 << 31, 2, WS, 256, None) == SHAPE
        assert lib.ip_linear_fp4(FAKE, 64, FAKE, FAKE, FAKE, 64, FAKE, FAKE, None, big, 4, 100, 50, FAKE, 50, 2, WS, 256, None) == PARAM
        assert lib.ip_fp4_block_bytes(4, big) == 0 and lib.ip_token_logprobs_workspace_bytes(4, big, 0) == 0


torch = pytest.importorskip("torch")
F, I8, U8 = torch.zeros(2, 64), torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2, 32, dtype=torch.uint8)
CALLS = (lambda: ip.quantize_fp4(F), lambda: ip.quantize_fp4(None), lambda: ip.rmsnorm_i8(F, F[0]), lambda: ip.rmsnorm_fp4(F, F[0], F),
         lambda: ip.dequantize_i8(I8, F[:, 0]), lambda: ip.dequantize_fp4(U8, U8, F[:, 0]), lambda: ip.linear_fp4(U8, U8, F, U8, U8, F),
         lambda: ip.token_logprobs(F), lambda: ip.token_logprobs([1.0]))


@pytest.mark.parametrize("i", range(len(CALLS)))
def test_the_calls_name_what_is_wrong(i):
    with pytest.raises(TypeError, match="CUDA tensor"):
        CALLS[i]()


@pytest.mark.parametrize("name,n", [("quantize_fp4", 4), ("linear_fp4", 11), ("rmsnorm_i8", 7), ("rmsnorm_fp4", 8), ("dequantize_i8", 4),
                                    ("dequantize_fp4", 6), ("token_logprobs", 5)])
def test_short_forms_take_nothing_but_plain_cuda_tensors(lib, name, n):
    f = getattr(ip._short, name)
    if ip._short is ip._Unbound:
        pytest.skip("no torch with CUDA to build for")
    for j in (None, 3, "x", 1.5, [1], object(), F, I8, U8, F[0, 0], torch.zeros(0), torch.float32):
        assert f(*[j] * n) is None
    for i in range(n):
        assert f(*[F if k != i else None for k in range(n)]) is None
    for m in (0, n - 1, n + 1):
        with pytest.raises(TypeError):
            f(*[None] * m)
