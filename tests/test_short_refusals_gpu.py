"""Refusals of the calls with run-time scales and on the 4-bit cache, each without and with a
workspace, so that the native short forms see them as well as the general ones; and single rows
of every layout against a contiguous copy."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ip():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_30846_gb300 as ip
    ip.load()
    return ip


def space(n=1 << 16):
    return torch.zeros(n, dtype=torch.uint8, device="cuda")


def refused(call, ok, cases):
    for err, over in cases:
        for ws in (None, space()):
            if "workspace" in over and ws is not None:
                continue
            with pytest.raises(err):
                call(**dict(dict(ok, workspace=ws), **over))


def test_rows_whose_elements_do_not_follow_one_another(ip):
    # all within their storage, also if they were read as consecutive bytes
    g = torch.Generator(device="cuda").manual_seed(1)
    base = torch.randint(-127, 128, (64, 64), generator=g, device="cuda", dtype=torch.int8)
    one = lambda *s: torch.ones(*s, device="cuda")
    bad = {"x row": base.t()[:1], "x vector": base.t()[0], "x step": base.view(1, -1)[:, :128:2],
           "x one byte": base[:1, :1].expand(1, 64), "x three": base.view(4, 16, 64)[:1, 2:3, ::2]}
    for x in bad.values():
        K = x.shape[-1]
        w = base[:5, :K].contiguous()
        with pytest.raises(ValueError):
            ip.linear_scaled_i8(x, one(x.shape[:-1]), w, one(5))
        with pytest.raises(ValueError):
            ip.linear_scaled_i8(x, one(x.shape[:-1]), w, one(5), workspace=space())
    for w in (base.t()[:1], base.view(1, -1)[:, :128:2], base[:1, :1].expand(1, 64)):
        for ws in (None, space()):
            with pytest.raises(ValueError):
                ip.linear_scaled_i8(base[:3], one(3), w, one(1), workspace=ws)


@pytest.mark.parametrize("K", [1, 16, 33, 64])
def test_single_rows_of_every_layout(ip, K):
    g = torch.Generator(device="cuda").manual_seed(K)
    base = torch.randint(-127, 128, (80, 80), generator=g, device="cuda", dtype=torch.int8)
    w = base[:7, :K]
    one = lambda *s: torch.ones(*s, device="cuda")
    rows = [base[3:4, :K], base[3, :K], base[2:3, 16:16 + K], base.view(5, 16, 80)[1:2, 4:5, :K]]
    if K == 1:
        rows += [base.t()[:1, :1], base[:1, ::80]]       # a last axis of one element has no stride
    for x in rows:
        for ws in (None, space()):
            y = ip.linear_scaled_i8(x, one(x.shape[:-1]), w, one(7), dtype=torch.float32, workspace=ws)
            want = x.double() @ w.double().t()
            assert torch.equal(y.double(), want)
            y = ip.linear_scaled_i8(w, one(7), x.reshape(1, K) if x.dim() != 2 else x, one(1), dtype=torch.float32,
                                    workspace=ws)
            assert torch.equal(y.double(), want.reshape(-1, 7).t())


def test_product_refusals_both_ways(ip):
    x = torch.zeros(4, 64, dtype=torch.int8, device="cuda")
    w, s4, s8 = torch.zeros(8, 64, dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda"), torch.ones(8, device="cuda")
    odd = torch.zeros(4, 65, dtype=torch.int8, device="cuda")
    refused(ip.linear_scaled_i8, dict(x=x, sx=s4, w=w, sw=s8), (
        (ValueError, dict(sx=s8)), (ValueError, dict(sw=s4)), (TypeError, dict(sx=s4.half())),
        (TypeError, dict(x=x.float())), (TypeError, dict(w=w.cpu())), (TypeError, dict(x=x.cpu())),
        (ValueError, dict(w=w[:, :48])), (ValueError, dict(w=w[0])), (ValueError, dict(bias=s4)),
        (TypeError, dict(bias=s8.cpu())), (TypeError, dict(dtype=torch.float64)), (ip.IpError, dict(x=odd[:, :64])),
        (ip.IpError, dict(x=odd[:, 1:])), (ip.IpError, dict(act=7)), (ip.IpError, dict(act=-1)),
        (ValueError, dict(x=x.t())), (ValueError, dict(x=x[:1].expand(4, 64))),
        (ValueError, dict(w=w[:1].expand(8, 64))), (ValueError, dict(sx=s8[::2])),
        (ValueError, dict(out=torch.zeros(4, 9, device="cuda"))),
        (TypeError, dict(out=torch.zeros(4, 8, device="cuda"), dtype=torch.float16)),
        (ValueError, dict(out=torch.zeros(8, 4, device="cuda").t())),
        (ValueError, dict(workspace=space(512)[::2])), (ip.IpError, dict(workspace=space(128))),
        (TypeError, dict(workspace=space().cpu()))))


def test_cache_refusals_both_ways(ip):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    q = torch.zeros(2, 1, 4, 128, device="cuda").half()
    k = torch.zeros(2, 3, 2, 128, device="cuda").half()
    cache, table, i2 = ip.kv4_cache(4, 2, 16), i32([[0], [1]]), i32([0, 1])
    shared = ((ValueError, dict(page_table=i32([[0]]))), (TypeError, dict(page_table=table.cpu())),
              (ValueError, dict(page_table=i32([[0, 1], [1, 0]]).t())), (ValueError, dict(page_table=i2)),
              (ValueError, dict(count=i32([1]))), (TypeError, dict(count=i2.long())), (ValueError, dict(cache=cache[:, :, :-1])),
              (TypeError, dict(cache=cache.to(torch.int8))), (ValueError, dict(cache=cache.transpose(0, 1))),
              (ip.IpError, dict(cache=torch.zeros(4, 2, 144 * 8, dtype=torch.uint8, device="cuda"))),
              (ip.IpError, dict(workspace=space(128))), (ValueError, dict(workspace=space(1024)[::2])))
    refused(ip.kv4_attention, dict(q=q, lengths=i2, page_table=table, cache=cache), shared + (
        (TypeError, dict(q=q.float())), (TypeError, dict(lengths=i2.long())), (TypeError, dict(lengths=None)),
        (ValueError, dict(lengths=i32([1]))), (ValueError, dict(q=q[..., ::2])), (ValueError, dict(q=q.transpose(2, 3))),
        (ip.IpError, dict(q=q[:, :, :3])), (ip.IpError, dict(scale=-1.0)), (ip.IpError, dict(scale=float("nan"))),
        (ip.IpError, dict(max_len=-1)), (ip.IpError, dict(q=q[:, :0])),
        (ip.IpError, dict(q=torch.zeros(2, 2049, 4, 128, device="cuda").half())),
        (ValueError, dict(out=torch.zeros(2, 1, 4, 64, device="cuda").half())), (TypeError, dict(out=q.float()))))
    refused(ip.kv4_append, dict(k=k, v=k, start=i2, page_table=table, cache=cache), shared + (
        (ValueError, dict(v=k[:, :2])), (TypeError, dict(v=k.float())), (TypeError, dict(start=None)),
        (ValueError, dict(k=k[:, :, :1], v=k[:, :, :1])), (TypeError, dict(k=k.int(), v=k.int())),
        (ValueError, dict(k=k[..., :64], v=k[..., :64])),
        (ValueError, dict(k=k.transpose(2, 3).contiguous().transpose(2, 3)))))
    refused(ip.kv4_read, dict(cache=cache, start=i2, page_table=table, T=2), shared + (
        (TypeError, dict(dtype=torch.float64)), (ValueError, dict(T=-1)), (TypeError, dict(start=None)),
        (TypeError, dict(start=i2.long()))))


def test_quantize_refusals(ip):
    x = torch.zeros(4, 64, device="cuda")
    for err, t in ((TypeError, x.int()), (TypeError, x.cpu()), (ValueError, x.t()), (ValueError, x[0].expand(3, 64)),
                   (ValueError, x[:1, ::2]), (ValueError, x[0, ::2]), (ValueError, x[:1, :1].expand(1, 64)),
                   (ValueError, torch.zeros(2, 3, 4, device="cuda").transpose(0, 1)),
                   (ValueError, torch.zeros(3, 0, device="cuda")), (ip.IpError, torch.zeros(1, 40000, device="cuda"))):
        with pytest.raises(err):
            ip.quantize_rows_i8(t)
    i8 = torch.zeros(4, 64, dtype=torch.int8, device="cuda")
    for err, kw in ((TypeError, dict(q=x)), (ValueError, dict(q=i8[:, :32])), (ValueError, dict(q=i8[:1].expand(4, 64))),
                    (TypeError, dict(scale=i8[:, 0])), (ValueError, dict(scale=x[0])), (TypeError, dict(scale=x[:, 0].cpu())),
                    (ValueError, dict(scale=x[:, 0]))):
        with pytest.raises(err):
            ip.quantize_rows_i8(x, **kw)
