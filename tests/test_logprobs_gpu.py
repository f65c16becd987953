"""Log probabilities, entropy and the best tokens on the GPU against float64: the tokens exactly,
the values to bounds of the f32 arithmetic."""
import math

import pytest

from guard import Guarded

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ip():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_30846_gb300 as ip
    ip.load()
    return ip


def reference(x, tokens, top, scale=1.0):
    """logprob, entropy, top log probabilities and tokens in float64, and what the bounds need."""
    V = x.shape[-1]
    a = x.double() * scale
    m = a.amax(1, keepdim=True)
    none = torch.isnan(a).any(1) | ~torch.isfinite(m[:, 0])
    d = torch.where(none[:, None], 0.0, a - m)
    e = torch.exp(d)
    s = e.sum(1)
    ls = torch.log(s)
    dd = torch.where(e > 0, d, 0.0)
    s1, s2 = (e * dd).sum(1).neg() / s, (e * dd * dd).sum(1) / s
    nan = lambda t: torch.where(none.view(-1, *[1] * (t.dim() - 1)), math.nan, t)
    lp = None
    if tokens is not None:
        t = tokens.long()
        lp = nan(d.gather(1, t.clamp(0, V - 1)[:, None])[:, 0] - ls)
        lp = torch.where(t < 0, 0.0, torch.where(t >= V, math.nan, lp))
    v, i = torch.sort(torch.where(none[:, None], 0.0, x.double() + 0.0), dim=1, descending=True, stable=True)
    tlp = nan((v[:, :top] * scale - torch.where(none[:, None], 0.0, m)) - ls[:, None])
    return lp, nan(ls + s1), tlp, torch.where(none[:, None], -1, i[:, :top]).int(), s1, s2


def check(ip, x, tokens=None, top=0, scale=1.0, **kw):
    lead, V = x.shape[:-1], x.shape[-1]
    flat = x.reshape(-1, V)
    lp, ent, tlp, ttok, s1, s2 = reference(flat, None if tokens is None else tokens.reshape(-1), top, scale)
    got = ip.token_logprobs(x, tokens, top=top, scale=scale, **kw)
    assert got[1].shape == lead and (got[0] is None) == (tokens is None) and (got[2] is None) == (got[3] is None) == (top == 0)
    # an exponential: three roundings of its argument and 2^-22; sums: up to 64 terms in turn, then a tree
    # and the parts; the logarithm, its argument's roundings: 84 steps of 2^-24 and what grows with |a - m|
    e_ls = U * (84 + 4 * s1)
    e_ent = e_ls + U * ((170 + 3 * s1) * s1 + 4 * s2) + U * (ent.abs().nan_to_num(0) + 2)
    near = lambda a, b, tol: bool((torch.isnan(a) == torch.isnan(b)).all() and (torch.isinf(a) == torch.isinf(b)).all() and
                                  ((a - b).abs().nan_to_num(0) <= tol).all())
    assert near(got[1].reshape(-1).double(), ent, e_ent)
    if tokens is not None:
        fin = lp.abs().nan_to_num(0, 0, 0)
        assert got[0].shape == lead and near(got[0].reshape(-1).double(), lp, e_ls + 4 * U * fin)
    if top:
        assert got[2].shape == got[3].shape == (*lead, top) and got[3].dtype == torch.int32
        assert torch.equal(got[3].reshape(-1, top), ttok)
        assert near(got[2].reshape(-1, top).double(), tlp, e_ls[:, None] + 4 * U * tlp.abs().nan_to_num(0, 0, 0))
    return got


def draw(rows, V, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = 3 * torch.randn(rows, V, generator=g, device="cuda") + 9 * (torch.rand(rows, V, generator=g, device="cuda") < 3 / V)
    return x.to(dtype), torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 2), (5, 31), (4, 32), (9, 33), (6, 257), (2, 504), (3, 505), (7, 1025), (2, 1272),
                                    (2, 1273), (3, 2040), (2, 2041), (3, 4088), (2, 4089), (2, 8184), (2, 8185), (1, 16384),
                                    (400, 9001), (1, 65536), (3, 131075), (1, 1 << 20)])
def test_matches_float64(ip, dtype, rows, V):
    x, tok = draw(rows, V, DT[dtype], V)
    for top in sorted({0, 1, min(V, 5), min(V, 32)}):
        check(ip, x, tok, top)


def test_many_rows(ip):
    x, tok = draw(12001, 1025, torch.bfloat16, 3)
    check(ip, x, tok, 5)
    x, tok = draw(3001, 70, torch.float16, 4)
    check(ip, x, tok.long(), 32, scale=0.7)


@pytest.mark.parametrize("V", [40, 1025, 5000, 30000, 131072])
def test_equal_sorted_and_masked_logits(ip, V):
    # equal logits, logits in order and all but a few ruled out: more tokens reach the bound than there is room for
    n = torch.arange(V, device="cuda").float()
    rows = [torch.zeros(V, device="cuda"), torch.full((V,), -1e30, device="cuda"), n, -n, (n / 100).floor(),
            torch.where(n % 2 == 0, 0.0, -0.0), torch.where(n > 3, -math.inf, n), torch.where(n == V - 1, 0.0, -math.inf),
            torch.where(n % 7 == 0, 5.0, -3.0), torch.where(n < 200, n, -math.inf)]
    x = torch.stack(rows)
    tok = torch.full((len(rows),), V - 1, device="cuda")
    for dtype in DT.values():
        y = x.clamp(max=60000).to(dtype) if dtype == torch.float16 else x.to(dtype)
        for top in (1, 20, 32):
            check(ip, y, tok, top)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [3, 100, 1025, 3000, 9001, 50000])
def test_rows_without_a_distribution(ip, dtype, V):
    x, tok = draw(8, V, DT[dtype], V)
    x[0, V - 1] = math.nan
    x[1, 0] = -math.nan
    x[2, V // 2] = math.inf
    x[3] = -math.inf
    x[4] = -math.inf
    x[4, V - 1] = math.nan
    x[5] = math.inf
    x[6] = -math.inf
    x[6, V // 2] = 2.0
    tok[3] = -1
    got = check(ip, x, tok, min(V, 7))
    assert got[0][3] == 0 and torch.isnan(got[1]).tolist() == [True] * 6 + [False] * 2 and got[1][6] == 0


def test_tokens_out_of_range(ip):
    for V in (50, 20000):
        x, _ = draw(6, V, torch.float32, 1)
        for dtype in (torch.int32, torch.int64):
            tok = torch.tensor([-1, -100, V, 2 ** 31 - 1, V - 1, 0], device="cuda", dtype=dtype)
            got = check(ip, x, tok, 2)
            assert got[0][:2].tolist() == [0, 0] and torch.isnan(got[0][2:4]).all()
        tok = torch.tensor([1 << 40, -(1 << 40), 1 << 32, (1 << 32) + 1, -(1 << 63), 5], device="cuda")
        assert torch.isnan(check(ip, x, tok)[0]).tolist() == [True, False, True, True, False, False]


@pytest.mark.parametrize("dtype", list(DT))
def test_rows_of_any_alignment(ip, dtype):
    base, _ = draw(4, 23000, DT[dtype], 6)
    for V in (20, 500, 1025, 2037, 2040, 4081, 8177, 8184, 16320):
        for at in range(9):
            x = base[:, at:at + V]
            check(ip, x, torch.full((4,), V - 1, device="cuda"), min(V, 9))
    x = base.view(2, 2, 23000)[:, :, 7:1032]
    tok = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    assert check(ip, x, tok, 3)[0].shape == (2, 2)
    assert check(ip, base[0, 3:900], torch.tensor(5, device="cuda"), 3)[1].dim() == 0
    assert ip.token_logprobs(base[:0], top=2)[3].shape == (0, 2)


def test_extreme_logits_and_scales(ip):
    x, tok = draw(5, 3000, torch.float32, 7)
    for k in (1e-30, 1e-3, 1e4, 1e30):
        check(ip, x * k, tok, 8)
    for scale in (1e-20, 0.1, 3.0, 1e10):
        check(ip, x, tok, 8, scale=scale)
    y = x.clone()
    y[:, 0], y[:, 1] = 3e38, -3e38
    check(ip, y, tok, 8)


def test_peaked_rows(ip):
    # all the weight on one token: log p and the entropy go to 0 from their own side
    x = torch.zeros(3, 2000, device="cuda")
    x[0, 7], x[1, 7], x[2, 7] = 20.0, 80.0, 200.0
    got = check(ip, x, torch.full((3,), 7, device="cuda"), 2)
    assert (got[0] <= 0).all() and (got[1] >= 0).all()


def test_outputs_workspace_and_streams(ip):
    rows, V, top = 3, 40000, 9
    x, tok = draw(rows, V, torch.bfloat16, 8)
    want = check(ip, x, tok, top)
    size = ip.token_logprobs_workspace_bytes(rows, V, top)
    ws = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    ws[:256] = 0
    f32, guards = torch.float32, [Guarded(s, t) for s, t in (((rows,), torch.float32), ((rows,), torch.float32),
                                                              ((rows, top), torch.float32), ((rows, top), torch.int32))]
    got = ip.token_logprobs(x, tok, top=top, out=tuple(g.view for g in guards), workspace=ws[:size])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (ws[size:] == 255).all() and ip.status(ws) == 0
    for g in guards:
        g.check()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    first = ip.token_logprobs(x, tok, top=top, stream=a)
    second = ip.token_logprobs(x, tok, top=top, stream=b)
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) and torch.equal(u, w) for u, v, w in zip(want, first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = ip.token_logprobs(x, tok, top=top, workspace=ws)
    x.copy_(x.flip(0))
    tok.copy_(tok.flip(0))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(u, v.flip(0)) for u, v in zip(kept, want))


def test_refusals(ip):
    x, tok = draw(4, 100, torch.float32, 1)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    f = ip.token_logprobs
    for err, call in ((TypeError, lambda: f(x.cpu())), (TypeError, lambda: f(x.double())), (TypeError, lambda: f(x, tok.float())),
                      (ValueError, lambda: f(x, tok[:3])), (ValueError, lambda: f(x.t())), (ip.IpError, lambda: f(x, top=33)),
                      (ip.IpError, lambda: f(x, top=-1)), (ip.IpError, lambda: f(x[:, :5].contiguous(), top=6)),
                      (ip.IpError, lambda: f(x, scale=0.0)), (ip.IpError, lambda: f(x, scale=math.nan)),
                      (ip.IpError, lambda: f(x, workspace=ws[:128])), (TypeError, lambda: f(x, workspace=x)),
                      (ip.IpError, lambda: f(torch.zeros(2, 200000, device="cuda"), workspace=ws)),
                      (ValueError, lambda: f(x, out=(None, x[0], None, None)))):
        with pytest.raises(err):
            call()
