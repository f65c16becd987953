"""The norm, the 4-bit rows, their product and the log probabilities as a decoder uses them: native short
forms against the general forms, a whole step eager and captured, on several streams."""
import pytest

from test_short_forms_gpu import both, ip  # noqa: F401 - a fixture

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import fp4_ref as ref


def some(r):
    return tuple(t for t in r if t is not None)


def comparable(r, rows, at):
    """Block scales without the bytes of rows behind the last, which are not written."""
    return tuple(torch.where(ref.untouched(t, rows), 0, t) if i == at else t for i, t in enumerate(r) if t is not None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 1024), (5, 33), (2, 3, 40), (7,), (0, 16), (3, 0, 16), (1, 1, 17), (4, 1, 9)])
def test_rows(ip, monkeypatch, dtype, shape):  # noqa: F811
    x = torch.randn(shape, device="cuda").to(dtype)
    r, g = torch.randn_like(x), torch.randn(shape[-1], device="cuda").to(dtype)
    rows = x.numel() // shape[-1]
    q, b, s = both(ip, monkeypatch, lambda: comparable(ip.quantize_fp4(x), rows, 1))
    assert ip.quantize_fp4(x)[0].stride(-1) == 1
    out = torch.empty_like(x)
    for kw in (dict(), dict(residual=r), dict(residual=r, out=out), dict(residual=r, eps=0.25)):
        both(ip, monkeypatch, lambda: some(ip.rmsnorm_i8(x, g, **kw)))
        both(ip, monkeypatch, lambda: comparable(ip.rmsnorm_fp4(x, g, **kw), rows, 1))
    both(ip, monkeypatch, lambda: some(ip.rmsnorm_i8(x, g, eps=1)), taken=False)
    q, b, s = ip.quantize_fp4(x)
    d, y = shape[-1], torch.empty(shape, device="cuda", dtype=dtype)
    for kw in (dict(), dict(d=d), dict(d=d, dtype=dtype), dict(d=d, out=y)):
        if kw.get("d") is not None or d % 2 == 0:
            both(ip, monkeypatch, lambda: ip.dequantize_fp4(q, b, s, **kw))
    q8, s8 = ip.quantize_rows_i8(x)
    for kw in (dict(), dict(dtype=dtype), dict(out=y)):
        both(ip, monkeypatch, lambda: ip.dequantize_i8(q8, s8, **kw))
    if len(shape) == 2 and shape[0] > 1:
        both(ip, monkeypatch, lambda: comparable(ip.quantize_fp4(x[:, 1:]), rows, 1), taken=False)
        both(ip, monkeypatch, lambda: some(ip.rmsnorm_i8(x[:, 1:], g[1:].clone())), taken=False)


@pytest.mark.parametrize("M,K,N", [(1, 64, 48), (1, 33, 1), (3, 40, 7), (200, 1000, 96), (0, 16, 4)])
def test_product(ip, monkeypatch, M, K, N):  # noqa: F811
    x, w = ip.quantize_fp4(torch.randn(M, K, device="cuda")), ip.quantize_fp4(torch.randn(N, K, device="cuda"))
    b, ws = torch.randn(N, device="cuda"), torch.zeros(256, dtype=torch.uint8, device="cuda")
    out = torch.empty(M, N, dtype=torch.float16, device="cuda")
    for kw in (dict(), dict(bias=b, act=ip.ACT_SWISH), dict(dtype=torch.float32), dict(out=out), dict(out=out, dtype=torch.float16)):
        both(ip, monkeypatch, lambda: ip.linear_fp4(*x, *w, workspace=ws, **kw))
    both(ip, monkeypatch, lambda: ip.linear_fp4(*x, *w), taken=False)
    for err, kw in ((TypeError, dict(dtype=torch.float64)), (ValueError, dict(bias=b[:0])), (ValueError, dict(out=out[:, :0])),
                    (TypeError, dict(out=out, dtype=torch.float32))):
        with pytest.raises(err):
            ip.linear_fp4(*x, *w, workspace=ws, **kw)
    if M:      # no rows: nothing is touched, the workspace neither
        for kw in (dict(workspace=ws[:128]), dict(workspace=ws, act=2)):
            with pytest.raises(ip.IpError):
                ip.linear_fp4(*x, *w, **kw)


@pytest.mark.parametrize("shape", [(3, 50), (1, 1025), (2, 3, 9000), (40,), (0, 100), (2, 200000)])
def test_logprobs(ip, monkeypatch, shape):  # noqa: F811
    x = torch.randn(shape, device="cuda").half()
    tok = torch.randint(0, shape[-1], shape[:-1], device="cuda")
    rows = x.numel() // shape[-1]
    for top in (0, 7):
        ws = torch.zeros(ip.token_logprobs_workspace_bytes(rows, shape[-1], top), dtype=torch.uint8, device="cuda")
        for kw in (dict(), dict(tokens=tok), dict(tokens=tok.int(), scale=0.5)):
            both(ip, monkeypatch, lambda: some(ip.token_logprobs(x, top=top, workspace=ws, **kw)))
    if rows:
        both(ip, monkeypatch, lambda: some(ip.token_logprobs(x, top=2)), taken=False)
        with pytest.raises(ip.IpError):
            ip.token_logprobs(x, top=33, workspace=ws)


@pytest.mark.parametrize("M", [1, 3, 600])
def test_outputs_lie_apart(ip, M):  # noqa: F811
    # small outputs of a call share an allocation: each starts on 16 bytes and is its own
    x, g = torch.randn(M, 1000, device="cuda").half(), torch.ones(1000, device="cuda").half()
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    calls = (lambda: ip.quantize_fp4(x), lambda: ip.rmsnorm_i8(x, g, x), lambda: ip.rmsnorm_fp4(x, g, x),
             lambda: ip.token_logprobs(x, torch.zeros(M, dtype=torch.int32, device="cuda"), top=3, workspace=ws))
    for call in calls:
        want, got = [t.clone() for t in call()], call()
        ends = sorted((t.data_ptr(), t.data_ptr() + (1 + sum((n - 1) * k for n, k in zip(t.shape, t.stride()))) * t.element_size()) for t in got)
        assert all(a[1] <= b[0] for a, b in zip(ends, ends[1:])) and all(a[0] % 16 == 0 for a in ends)
        for i, t in enumerate(got):
            t.zero_()
            assert all(torch.equal(u, v) for u, v in list(zip(got, want))[i + 1:] if u.dim() != 3)


class Step:
    """A decoder's feed-forward block and head on M tokens: norm with residual into 4-bit rows, two 4-bit
    products, norm into int8, the head's product, log probabilities with the best tokens."""

    def __init__(self, ip, M, seed=0):  # noqa: F811
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *n: torch.randn(*n, generator=g, device="cuda")
        self.ip, self.M = ip, M
        self.up, self.down = ip.quantize_fp4(rnd(2048, 512) / 22), ip.quantize_fp4(rnd(512, 2048) / 45)
        self.head, self.head_scale = ip.quantize_rows_i8(rnd(1025, 512) / 8)
        self.g1, self.g2, self.bias = 1 + 0.1 * rnd(512), 1 + 0.1 * rnd(512), rnd(2048)
        self.g1, self.g2 = self.g1.bfloat16(), self.g2.bfloat16()
        self.x, self.res = rnd(M, 512).bfloat16(), 2 * rnd(M, 512).bfloat16()
        self.tokens = torch.randint(0, 1025, (M,), generator=g, device="cuda")
        self.ws = torch.zeros(256, dtype=torch.uint8, device="cuda")

    def run(self):
        ip, ws = self.ip, self.ws  # noqa: F811
        q, b, s, h = ip.rmsnorm_fp4(self.x, self.g1, self.res)
        mid = ip.linear_fp4(q, b, s, *self.up, self.bias, act=ip.ACT_SWISH, workspace=ws)
        y = ip.linear_fp4(*ip.quantize_fp4(mid), *self.down, workspace=ws)
        q8, s8, h2 = ip.rmsnorm_i8(y, self.g2, h)
        logits = ip.linear_scaled_i8(q8, s8, self.head, self.head_scale, dtype=torch.float32, workspace=ws)
        return (h, mid, y, h2, logits, *ip.token_logprobs(logits, self.tokens, top=4, workspace=ws))


@pytest.mark.parametrize("M", [1, 7, 130, 1000])
def test_a_step(ip, M):  # noqa: F811
    st = Step(ip, M)
    h, mid, y, h2, logits, lp, ent, tlp, ttok = st.run()
    assert ip.status(st.ws) == 0
    # each stage in float64 from what the one before gave: its own roundings only, bf16 has eight bits and rounds by
    # 2^-8 of a value at most; the sums in f32 are far below that
    assert torch.equal(h, st.x + st.res)
    z = (h.double() * st.g1.double())
    c, sb, r = ref.quantize(z)
    q, b = ref.bytes_of(c, sb)
    rows = ref.values(q, b, r, 512) * (h.double().square().mean(1, keepdim=True) + 1e-5).rsqrt()
    pre = rows @ ref.values(*st.up, 512).t() + st.bias.double()
    want = pre * torch.sigmoid(pre)
    assert ((mid.double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.01 + 2.0 ** -12).all()
    c, sb, r = ref.quantize(mid)
    want = ref.values(*ref.bytes_of(c, sb), r, 2048) @ ref.values(*st.down, 2048).t()
    assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.01 + 2.0 ** -12).all()
    assert torch.equal(h2, h + y)
    z = h2.double() * st.g2.double()
    top = z.abs().amax(1, keepdim=True)
    rows = (127 * z / top).round() * (top / 127) * (h2.double().square().mean(1, keepdim=True) + 1e-5).rsqrt()
    want = rows @ (st.head.double() * st.head_scale.double()[:, None]).t()
    assert ((logits.double() - want).abs() <= 2.0 ** -18 * (rows.abs() @ (st.head.double() * st.head_scale.double()[:, None]).abs().t())).all()
    ls = torch.log_softmax(logits.double(), 1)
    assert torch.allclose(lp.double(), ls.gather(1, st.tokens[:, None])[:, 0], rtol=0, atol=1e-5)
    assert torch.equal(ttok[:, 0].long(), logits.argmax(1)) and torch.allclose(tlp.double(), ls.gather(1, ttok.long()), rtol=0, atol=1e-5)
    assert torch.allclose(ent.double(), -(ls.exp() * ls).sum(1), rtol=0, atol=1e-4)


def test_steps_captured_replayed_and_on_two_streams(ip):  # noqa: F811
    a, b = Step(ip, 64, 1), Step(ip, 200, 2)
    want = [[t.clone() for t in s.run()] for s in (a, b)]
    graphs, outs = [], []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
    for _ in range(3):      # two captured graphs, one after the other, and at once on two streams
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(o, w))
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in graphs]
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(o, w))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = a.run()
    mine = b.run()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(other, want[0])) and all(torch.equal(x, y) for x, y in zip(mine, want[1]))
    assert ip.status(a.ws) == 0 and ip.status(b.ws) == 0
