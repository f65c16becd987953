"""Native short forms against the general forms: same bits, same refusals."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ip():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_30846_gb300 as ip
    ip.load()
    assert ip._short is not ip._Unbound
    return ip


class Spy:
    """The short forms, noting whether each call was taken."""

    def __init__(self, short):
        self.short, self.taken = short, []

    def __getattr__(self, name):
        def call(*args):
            r = getattr(self.short, name)(*args)
            self.taken.append(r is not None)
            return r
        return call


def both(ip, monkeypatch, call, taken=True):
    """Results of the call by the short and by the general form, bit for bit alike."""
    spy = Spy(ip._short)
    res = []
    for short in (spy, ip._Unbound):
        with monkeypatch.context() as m:
            m.setattr(ip, "_short", short)
            r = call()
        res.append([t.clone() for t in (r if isinstance(r, tuple) else (r,))])
    assert spy.taken == [taken]
    for a, b in zip(*res):
        assert a.dtype == b.dtype and a.shape == b.shape and a.device == b.device
        assert torch.equal(torch.nan_to_num(a.float(), 7.0), torch.nan_to_num(b.float(), 7.0))
    return res[0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 1024), (5, 33), (2, 3, 40), (7,), (0, 16), (3, 0, 16), (1, 1, 17), (4, 1, 9)])
def test_quantize(ip, monkeypatch, dtype, shape):
    x = torch.randn(shape, device="cuda").to(dtype)
    q, s = both(ip, monkeypatch, lambda: ip.quantize_rows_i8(x))
    q1, _ = ip.quantize_rows_i8(x)
    if q1.dim() > 1 and q1.numel() and q1.shape[-2] > 1:
        assert q1.stride(-2) % 16 == 0
    oq, os = torch.empty_like(q), torch.empty_like(s)
    both(ip, monkeypatch, lambda: ip.quantize_rows_i8(x, q=oq, scale=os))
    assert ip.quantize_rows_i8(x, q=oq, scale=os)[0] is oq or torch.equal(oq, q)
    if len(shape) == 2 and shape[0] > 1:
        both(ip, monkeypatch, lambda: ip.quantize_rows_i8(x[:, 1:]), taken=False)


@pytest.mark.parametrize("M,K,N", [(1, 64, 48), (1, 33, 1), (3, 40, 7), (200, 1000, 96), (0, 16, 4)])
def test_product(ip, monkeypatch, M, K, N):
    q, s = ip.quantize_rows_i8(torch.randn(M, K, device="cuda"))
    w, sw = ip.quantize_rows_i8(torch.randn(N, K, device="cuda"))
    b, ws = torch.randn(N, device="cuda"), torch.zeros(256, dtype=torch.uint8, device="cuda")
    out = torch.empty(M, N, dtype=torch.float16, device="cuda")
    for kw in (dict(), dict(bias=b, act=ip.ACT_SWISH), dict(dtype=torch.float32), dict(out=out),
               dict(out=out, dtype=torch.float16)):
        both(ip, monkeypatch, lambda: ip.linear_scaled_i8(q, s, w, sw, workspace=ws, **kw))
    if M > 1:
        lead = q.view(1, *q.shape) if q.is_contiguous() else None
        if lead is not None and K % 16 == 0:
            both(ip, monkeypatch, lambda: ip.linear_scaled_i8(lead, s[None], w, sw, workspace=ws))
    both(ip, monkeypatch, lambda: ip.linear_scaled_i8(q, s, w, sw), taken=False)
    for err, kw in ((TypeError, dict(dtype=torch.float64)), (ip.IpError, dict(act=2)), (ValueError, dict(bias=b[:0])),
                    (ValueError, dict(out=out[:, :0])), (TypeError, dict(out=out, dtype=torch.float32))):
        if kw.get("act") == 2 and M == 0:
            continue
        with pytest.raises(err):
            ip.linear_scaled_i8(q, s, w, sw, workspace=ws, **kw)
    if M:      # no rows: nothing is touched, the workspace neither
        with pytest.raises(ip.IpError):
            ip.linear_scaled_i8(q, s, w, sw, workspace=ws[:128])


def test_cache(ip, monkeypatch):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cache, table = ip.kv4_cache(8, 2, 16), i32([[3, 1, 6], [0, 7, 2]])
    kv = torch.randn(2, 40, 3, 2, 128, device="cuda").half()
    k, v = kv[:, :, 0], kv[:, :, 1]
    start, count, lens = i32([0, 1]), i32([40, 30]), i32([40, 31])
    ws = torch.zeros(ip.kv4_attention_workspace_bytes(2, 3, 4, 2, 48), dtype=torch.uint8, device="cuda")
    both(ip, monkeypatch, lambda: ip.kv4_append(k, v, start, table, cache, count=count, workspace=ws))
    for c in (None, count):
        both(ip, monkeypatch, lambda: ip.kv4_read(cache, start, table, 40, count=c, dtype=torch.float32, workspace=ws))
    q = torch.randn(2, 3, 4, 128, device="cuda").half()
    out = torch.empty_like(q)
    for kw in (dict(), dict(causal=False), dict(scale=0.3), dict(max_len=45), dict(count=i32([3, 1])), dict(out=out)):
        both(ip, monkeypatch, lambda: ip.kv4_attention(q, lens, table, cache, workspace=ws, **kw))
    both(ip, monkeypatch, lambda: ip.kv4_attention(q, lens, table, cache), taken=False)
    both(ip, monkeypatch, lambda: ip.kv4_attention(q, lens, table, cache, scale=1, workspace=ws), taken=False)
    assert ip.status(ws) == 0
    for kw in (dict(scale=-1.0), dict(max_len=-1), dict(workspace=ws[:200])):
        with pytest.raises(ip.IpError):
            ip.kv4_attention(q, lens, table, cache, **dict(dict(workspace=ws), **kw))
    with pytest.raises(ValueError):
        ip.kv4_attention(q, lens, table, cache, out=out[:, :1], workspace=ws)
    with pytest.raises(ip.IpError):
        ip.kv4_append(k, v, start, table, cache, workspace=ws[:128])
    with pytest.raises(TypeError):
        ip.kv4_read(cache, start, table, 4, dtype=torch.float64, workspace=ws)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = ip.kv4_attention(q, lens, table, cache, workspace=ws)
    side.synchronize()
    assert torch.equal(got, ip.kv4_attention(q, lens, table, cache, workspace=ws, stream=torch.cuda.current_stream()))
