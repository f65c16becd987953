"""Refusals of the operators with run-time scales and of the 4-bit cache, without a
GPU: every case fails validation before any pointer is used."""
import ctypes

import pytest

import paper_2609_30846_gb300 as ip

P = ctypes.c_void_p
FAKE, WS = P(1 << 20), P(1 << 21)
STR = (ctypes.c_longlong * 3)(1024, 128, 128)
NULL, SHAPE, ALIGN, UNSUPPORTED, PARAM, WORKSPACE = -1, -2, -3, -4, -7, -8


@pytest.fixture(scope="module")
def lib():
    return ip.load()


def call(fn, order, base, **over):
    a = dict(base, **over)
    return fn(*[a[n] for n in order])


def test_quantize_refusals(lib):
    order = ("x", "dtype", "rows", "d", "ldx", "q", "ldq", "scale", "stream")
    base = dict(x=FAKE, dtype=2, rows=4, d=100, ldx=100, q=FAKE, ldq=112, scale=FAKE, stream=None)
    run = lambda **o: call(lib.ip_quantize_rows_i8, order, base, **o)
    assert run(rows=0, x=None, q=None, scale=None) == 0
    for over, code in ((dict(dtype=3), PARAM), (dict(dtype=-1), PARAM), (dict(rows=-1), SHAPE),
                       (dict(rows=(1 << 40) + 1), SHAPE), (dict(d=0), SHAPE), (dict(d=32769, ldx=40000, ldq=40000), SHAPE),
                       (dict(ldx=99), SHAPE), (dict(ldq=99), SHAPE), (dict(x=None), NULL), (dict(q=None), NULL),
                       (dict(scale=None), NULL), (dict(x=P((1 << 20) + 1)), ALIGN),
                       (dict(dtype=0, x=P((1 << 20) + 2)), ALIGN), (dict(scale=P((1 << 20) + 2)), ALIGN)):
        assert run(**over) == code, over


def test_linear_scaled_refusals(lib):
    order = ("x", "ldx", "sx", "w", "ldw", "sw", "bias", "act", "rows", "K", "N", "y", "ldy", "dtype", "ws", "wsb",
             "stream")
    base = dict(x=FAKE, ldx=112, sx=FAKE, w=FAKE, ldw=112, sw=FAKE, bias=None, act=0, rows=4, K=100, N=50, y=FAKE,
                ldy=50, dtype=2, ws=WS, wsb=256, stream=None)
    run = lambda **o: call(lib.ip_linear_scaled_i8, order, base, **o)
    assert run(rows=0, x=None, w=None, y=None, ws=None) == 0
    for over, code in ((dict(dtype=3), PARAM), (dict(act=2), PARAM), (dict(act=-1), PARAM), (dict(rows=-1), SHAPE),
                       (dict(rows=(1 << 27) + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=32769, ldx=32784, ldw=32784), SHAPE),
                       (dict(N=0), SHAPE), (dict(N=65537, ldy=65537), SHAPE), (dict(ldx=96), SHAPE),
                       (dict(ldw=96), SHAPE), (dict(ldy=49), SHAPE), (dict(ldx=1 << 41), SHAPE),
                       (dict(x=None), NULL), (dict(sx=None), NULL), (dict(w=None), NULL), (dict(sw=None), NULL),
                       (dict(y=None), NULL), (dict(ws=None), NULL), (dict(ldx=104), ALIGN), (dict(ldw=101), ALIGN),
                       (dict(x=P((1 << 20) + 8)), ALIGN), (dict(w=P((1 << 20) + 1)), ALIGN),
                       (dict(sx=P((1 << 20) + 2)), ALIGN), (dict(sw=P((1 << 20) + 1)), ALIGN),
                       (dict(bias=P((1 << 20) + 3)), ALIGN), (dict(y=P((1 << 20) + 1)), ALIGN),
                       (dict(dtype=0, y=P((1 << 20) + 2)), ALIGN), (dict(ws=P((1 << 21) + 16)), ALIGN),
                       (dict(wsb=255), WORKSPACE)):
        assert run(**over) == code, over


CACHE = dict(table=FAKE, width=4, cache=FAKE, pages=9, page=32, ws=WS, wsb=256, stream=None)
CACHE_REFUSALS = ((dict(dh=64), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(page=128), UNSUPPORTED),
                  (dict(page=0), UNSUPPORTED), (dict(width=0), SHAPE), (dict(width=1 << 24), SHAPE),
                  (dict(pages=-1), SHAPE), (dict(table=None), NULL), (dict(cache=None), NULL), (dict(ws=None), NULL),
                  (dict(table=P((1 << 20) + 2)), ALIGN), (dict(cache=P((1 << 20) + 8)), ALIGN),
                  (dict(ws=P((1 << 21) + 64)), ALIGN), (dict(wsb=255), WORKSPACE))


def test_page_bytes(lib):
    for page in (16, 32, 64):
        assert ip.kv4_page_bytes(page) == 144 * page
    for page, dh in ((0, 128), (8, 128), (48, 128), (128, 128), (16, 64)):
        assert lib.ip_kv4_page_bytes(page, dh) == 0
    with pytest.raises(ip.IpError):
        ip.kv4_page_bytes(24)


def test_append_refusals(lib):
    order = ("k", "v", "dtype", "ks", "vs", "start", "count", "B", "T", "H", "dh", "table", "width", "cache", "pages",
             "page", "ws", "wsb", "stream")
    base = dict(CACHE, k=FAKE, v=FAKE, dtype=1, ks=STR, vs=STR, start=FAKE, count=None, B=2, T=3, H=8, dh=128)
    run = lambda **o: call(lib.ip_kv4_append, order, base, **o)
    assert run(B=0, k=None, cache=None) == 0 and run(T=0, k=None, cache=None) == 0
    neg = (ctypes.c_longlong * 3)(1024, -1, 128)
    far = (ctypes.c_longlong * 3)((1 << 40) + 1, 0, 0)
    for over, code in CACHE_REFUSALS + (
            (dict(dtype=4), PARAM), (dict(B=-1), SHAPE), (dict(B=65536), SHAPE), (dict(T=-1), SHAPE),
            (dict(B=65535, T=65535), SHAPE), (dict(H=0), SHAPE), (dict(H=65536), SHAPE), (dict(k=None), NULL),
            (dict(v=None), NULL), (dict(start=None), NULL), (dict(ks=None), NULL), (dict(vs=None), NULL),
            (dict(ks=neg), SHAPE), (dict(vs=far), SHAPE), (dict(k=P((1 << 20) + 1)), ALIGN),
            (dict(dtype=0, v=P((1 << 20) + 2)), ALIGN), (dict(start=P((1 << 20) + 2)), ALIGN),
            (dict(count=P((1 << 20) + 2)), ALIGN)):
        assert run(**over) == code, over


def test_read_refusals(lib):
    order = ("cache", "pages", "page", "table", "width", "start", "count", "B", "T", "H", "dh", "k", "v", "dtype",
             "ws", "wsb", "stream")
    base = dict(CACHE, start=FAKE, count=None, B=2, T=3, H=8, dh=128, k=FAKE, v=FAKE, dtype=0)
    run = lambda **o: call(lib.ip_kv4_read, order, base, **o)
    assert run(B=0, k=None, cache=None) == 0
    for over, code in CACHE_REFUSALS + (
            (dict(dtype=3), PARAM), (dict(B=65536), SHAPE), (dict(T=-1), SHAPE), (dict(k=None), NULL),
            (dict(v=None), NULL), (dict(start=None), NULL), (dict(k=P((1 << 20) + 8)), ALIGN),
            (dict(count=P((1 << 20) + 1)), ALIGN)):
        assert run(**over) == code, over


def test_attention_refusals(lib):
    order = ("q", "dtype", "qs", "lengths", "count", "causal", "scale", "B", "T", "H", "Hkv", "dh", "max_len", "table",
             "width", "cache", "pages", "page", "out", "ws", "wsb", "stream")
    base = dict(CACHE, q=FAKE, dtype=2, qs=STR, lengths=FAKE, count=None, causal=1, scale=0.1, B=2, T=3, H=8, Hkv=2,
                dh=128, max_len=64, out=FAKE, wsb=1 << 24)
    run = lambda **o: call(lib.ip_kv4_attention, order, base, **o)
    assert run(B=0, q=None, cache=None, out=None) == 0
    for over, code in CACHE_REFUSALS + (
            (dict(dtype=0), PARAM), (dict(causal=2), PARAM), (dict(scale=0.0), PARAM), (dict(scale=-1.0), PARAM),
            (dict(scale=float("nan")), PARAM), (dict(scale=float("inf")), PARAM), (dict(B=-1), SHAPE),
            (dict(T=0), SHAPE), (dict(T=2049), SHAPE), (dict(H=7), SHAPE), (dict(Hkv=0), SHAPE), (dict(H=0), SHAPE),
            (dict(max_len=-1), SHAPE), (dict(max_len=(1 << 28) + 1), SHAPE), (dict(q=None), NULL),
            (dict(qs=None), NULL), (dict(lengths=None), NULL), (dict(out=None), NULL), (dict(q=P((1 << 20) + 1)), ALIGN),
            (dict(out=P((1 << 20) + 8)), ALIGN), (dict(lengths=P((1 << 20) + 2)), ALIGN),
            (dict(count=P((1 << 20) + 2)), ALIGN)):
        assert run(**over) == code, over
    need = ip.kv4_attention_workspace_bytes(2, 3, 8, 2, 64)
    assert run(wsb=need - 1) == WORKSPACE


def test_attention_workspace_covers_its_plan():
    # the status word, and for one wave of CTAs two partial rows each; shapes out of range have none
    assert ip.kv4_attention_workspace_bytes(1, 1, 1, 1, 1) == 256
    for B, T, H, Hkv, n in ((1, 1, 8, 8, 375), (64, 1, 32, 8, 8192), (1, 1, 1, 1, 1 << 28), (65535, 1, 8, 1, 4096),
                            (4, 33, 8, 8, 1500), (1, 2048, 64, 1, 100000), (0, 1, 8, 8, 10), (3, 1, 8, 8, 0)):
        size = ip.kv4_attention_workspace_bytes(B, T, H, Hkv, n)
        assert 256 <= size <= 1 << 23 and size % 256 == 0
    for bad in ((1, 0, 8, 8, 10), (1, 1, 8, 3, 10), (1, 1, 0, 1, 10), (1, 1, 8, 8, -1), (-1, 1, 8, 8, 10)):
        with pytest.raises(ip.IpError):
            ip.kv4_attention_workspace_bytes(*bad)


def test_binding_takes_cuda_tensors_only():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4, 8, 128)
    i8, i32 = torch.zeros(2, 16, dtype=torch.int8), torch.zeros(2, dtype=torch.int32)
    for call_ in (lambda: ip.quantize_rows_i8(x), lambda: ip.linear_scaled_i8(i8, x, i8, x),
                  lambda: ip.kv4_append(x, x, i32, i32, i8), lambda: ip.kv4_read(i8, i32, i32, 4),
                  lambda: ip.kv4_attention(x.half(), i32, i32, i8)):
        with pytest.raises(TypeError):
            call_()
