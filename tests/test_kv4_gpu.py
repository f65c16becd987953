"""The 4-bit key/value cache on the GPU: append and read bit for bit against the
definition, the attention against 64 bits within a derived bound."""
import numpy as np
import pytest

import kv4_ref as ref
from guard import Guarded

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ip():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_30846_gb300 as ip
    ip.load()
    return ip


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def f64(t):
    return t.double().cpu().numpy()


def space(n=256):
    return torch.zeros(n, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------ append and read

@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("B,T,H", [(1, 1, 1), (3, 1, 8), (2, 17, 3), (2, 70, 2)])
def test_append_writes_the_definition(ip, dtype, page, B, T, H):
    rng = np.random.default_rng(B * 100 + T + page)
    g = torch.Generator(device="cuda").manual_seed(T)
    k, v = (torch.randn(B, T, H, 128, generator=g, device="cuda").mul(4).to(DT[dtype]) for _ in range(2))
    start = [int(x) for x in rng.integers(0, 3 * page, B)]
    count = [T] + [int(x) for x in rng.integers(0, T + 1, B - 1)]
    width = -(-(max(start) + T) // page)
    ids = rng.permutation(B * width + 2)[:B * width].reshape(B, width).astype(np.int32)
    cache = ip.kv4_cache(B * width + 2, H, page)
    cache.fill_(0xa5)
    want = cache.cpu().numpy().copy()
    ws = space()
    ip.kv4_append(k, v, ints(start), torch.from_numpy(ids).cuda(), cache, count=ints(count), workspace=ws)
    parts = (*ref.rows_bytes(f64(k), ref.K_BYTE), *ref.rows_bytes(f64(v), ref.V_BYTE))
    for b in range(B):
        for t in range(count[b]):
            pos = start[b] + t
            base = 0
            for part, size in zip(parts, (64, 8, 64, 8)):
                o = base + pos % page * size
                want[ids[b, pos // page], :, o:o + size] = part[b, t]
                base += size * page
    assert ip.status(ws) == 0
    np.testing.assert_array_equal(cache.cpu().numpy(), want)
    for out in ("f32", dtype):
        ko, vo = ip.kv4_read(cache, ints(start), torch.from_numpy(ids).cuda(), T, count=ints(count),
                             dtype=DT[out], workspace=ws)
        for got, x in ((ko, k), (vo, v)):
            val = torch.from_numpy(ref.values(f64(x))).float().to(DT[out])
            for b in range(B):
                val[b, count[b]:] = 0
            assert torch.equal(got.cpu(), val)
    assert ip.status(ws) == 0


def test_append_values_at_the_borders(ip):
    # ties between codes and their neighbours, scales on the middle of two bf16 values,
    # subnormal and huge groups, zeros, NaN and infinities
    rows = []
    for s in (1.0, 0.3, 1.5e-3, 2.0 ** -120, 3e37):
        s = float(ref.round_bf16(np.float64(s)))
        t = np.array([(i + 0.5) * s for i in range(8)] + [7 * s], np.float32)
        t = np.concatenate([t, np.nextafter(t, np.float32(0)), np.nextafter(t, np.float32(np.inf))])
        t = t[np.abs(t) <= 7 * s]
        r = np.zeros(128, np.float32)
        r[:t.size], r[64:64 + t.size] = t, -t
        r[[31, 63, 95, 127]] = 7 * s
        rows.append(r)
    mid = (np.arange(128, 256) + 0.5) / 128 * 7
    for f in (1.0, 2.0 ** -100, 2.0 ** 100):
        for j in range(0, 128, 4):
            r = np.zeros(128, np.float32)
            for i in range(4):
                x = np.float32(mid[j + i] * f)
                r[32 * i] = (x, np.nextafter(x, np.float32(0)), np.nextafter(x, np.float32(np.inf)), -x)[j // 4 % 4]
                r[32 * i + 1] = x / 3
            rows.append(r)
    for f in (1e-45, 1e-40, 7e-39, 1.2e-38, 3e38):
        rows.append((np.random.default_rng(1).uniform(-1, 1, 128) * f).astype(np.float32))
    rows.append(np.zeros(128, np.float32))
    for bad in (np.nan, np.inf, -np.inf):
        r = np.linspace(-1, 1, 128).astype(np.float32)
        r[40] = bad
        rows.append(r)
    x = np.stack(rows)[None, :, None]
    T = x.shape[1]
    k = torch.from_numpy(x).cuda()
    width = -(-T // 16)
    cache = ip.kv4_cache(width, 1, 16)
    table = torch.arange(width, dtype=torch.int32, device="cuda")[None]
    ip.kv4_append(k, -k, ints([0]), table, cache)
    ko, vo = ip.kv4_read(cache, ints([0]), table, T, dtype=torch.float32)
    np.testing.assert_array_equal(f64(ko), ref.values(x.astype(np.float64)))
    np.testing.assert_array_equal(f64(vo), ref.values(-x.astype(np.float64)))


def test_append_strided_views_of_a_stacked_projection(ip):
    B, T, H = 2, 9, 4
    qkv = torch.randn(B, T, 3 * H * 128 + 1, device="cuda").to(torch.bfloat16)[..., 1:]   # odd base
    k, v = (qkv[..., i * H * 128:(i + 1) * H * 128].unflatten(-1, (H, 128)) for i in (1, 2))
    cache = ip.kv4_cache(2, H, 32)
    table = ints([[1], [0]])
    ip.kv4_append(k, v, ints([0, 5]), table, cache)
    ko, vo = ip.kv4_read(cache, ints([0, 5]), table, T, dtype=torch.float32)
    np.testing.assert_array_equal(f64(ko), ref.values(f64(k)))
    np.testing.assert_array_equal(f64(vo), ref.values(f64(v)))
    kt = torch.randn(B, H, T, 128, device="cuda").transpose(1, 2)      # head-split memory
    ip.kv4_append(kt, kt, ints([0, 5]), table, cache)
    ko, vo = ip.kv4_read(cache, ints([0, 5]), table, T, dtype=torch.float32)
    np.testing.assert_array_equal(f64(ko), ref.values(f64(kt)))
    np.testing.assert_array_equal(f64(vo), ref.values(f64(kt)))


def test_pages_and_positions_that_do_not_exist(ip):
    k = torch.randn(4, 20, 2, 128, device="cuda")
    cache = ip.kv4_cache(3, 2, 16)
    before = cache.clone()
    table = ints([[0, 7], [-1, 1], [2, 1], [2, 1]])
    ws = space()
    # sequence 0 ends in a page past the cache, 1 begins in none, 2 runs past the table, 3 begins
    # before it
    ip.kv4_append(k, k, ints([0, 0, 30, -8]), table, cache, count=ints([20, 20, 4, 3]), workspace=ws)
    assert ip.status(ws) == -7
    assert ip.status(ws) == 0
    want = ip.kv4_cache(3, 2, 16)
    want.copy_(before)
    ip.kv4_append(k[:1, :16], k[:1, :16], ints([0]), ints([[0]]), want)
    ip.kv4_append(k[1:2, 16:], k[1:2, 16:], ints([0]), ints([[1]]), want)
    ip.kv4_append(k[2:3, :2], k[2:3, :2], ints([14]), ints([[1]]), want)
    assert torch.equal(cache, want)
    ko, vo = ip.kv4_read(cache, ints([0, 0, 30, -8]), table, 20, count=ints([20, 20, 4, 3]), workspace=ws)
    assert ip.status(ws) == -7
    assert not ko[0, 16:].any() and not ko[1, :16].any() and not ko[2, 2:].any() and not ko[3].any()
    assert ko[0, :16].any() and ko[1, 16:].any() and ko[2, :2].any()


# ------------------------------------------------------------ attention

def make(B, T, H, Hkv, lens, page, dtype, seed, kscale=1.0, qscale=1.5):
    rng = np.random.default_rng(seed)
    ks = [rng.standard_normal((n, Hkv, 128)) * kscale * (1 + 3 * (rng.random((Hkv, 128)) < 0.03)) for n in lens]
    vs = [rng.standard_normal((n, Hkv, 128)) for n in lens]
    cache, table = ref.build_cache(ks, vs, page, rng)
    q = torch.from_numpy(rng.standard_normal((B, T, H, 128)) * qscale).to(DT[dtype]).cuda()
    return q, ks, vs, torch.from_numpy(cache).cuda(), torch.from_numpy(table).cuda()


def check(ip, got, q, ks, vs, counts, causal, scale=128 ** -0.5):
    want, bound = ref.attention(f64(q), ks, vs, counts, causal, scale)
    fin = torch.finfo(q.dtype)
    tol = bound * (1 + fin.eps) + np.abs(want) * fin.eps / 2 + fin.smallest_normal * fin.eps
    err = np.abs(f64(got) - want)
    assert np.isfinite(f64(got)).all()
    assert (err <= tol).all(), (float(err.max()), float((err / tol).max()))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("B,T,H,Hkv,lens", [
    (1, 1, 1, 1, [1]), (1, 1, 8, 8, [375]), (2, 1, 4, 2, [16, 17]), (3, 1, 8, 1, [0, 63, 1000]),
    (2, 1, 12, 4, [65, 64]), (1, 1, 20, 2, [301]), (2, 3, 4, 4, [40, 3]), (2, 5, 6, 2, [5, 129]),
    (1, 33, 3, 3, [200]), (1, 9, 16, 2, [9])])
def test_attention(ip, dtype, page, B, T, H, Hkv, lens):
    q, ks, vs, cache, table = make(B, T, H, Hkv, lens, page, dtype, seed=B + T + H + sum(lens) + page)
    for causal in (True, False):
        ws = space(ip.kv4_attention_workspace_bytes(B, T, H, Hkv, max(lens) + 5))
        out = Guarded((B, T, H, 128), DT[dtype])
        got = ip.kv4_attention(q, ints(lens), table, cache, causal=causal, max_len=max(max(lens), 1), out=out.view,
                               workspace=ws)
        assert ip.status(ws) == 0
        check(ip, got, q, ks, vs, [T] * B, causal)
        out.check()


@pytest.mark.parametrize("T,counts,lens", [(4, [4, 0, 2, 1], [9, 9, 2, 0]), (6, [6, 6, 3, 9], [2, 6, 1, 40]),
                                           (20, [1, 20, 7, 13], [70, 20, 90, 13])])
def test_ragged_counts_and_empty_rows(ip, T, counts, lens):
    # sequences with more queries than tokens leave their first queries without a key
    q, ks, vs, cache, table = make(4, T, 4, 2, lens, 16, "bf16", seed=T)
    for causal in (True, False):
        ws = space(ip.kv4_attention_workspace_bytes(4, T, 4, 2, 100))
        got = ip.kv4_attention(q, ints(lens), table, cache, count=ints(counts), causal=causal, max_len=100,
                               workspace=ws)
        assert ip.status(ws) == 0
        c = [min(x, T) for x in counts]
        check(ip, got, q, ks, vs, c, causal)
        for b in range(4):
            assert not got[b, c[b]:].any()
            if causal and c[b] > lens[b]:
                assert not got[b, :c[b] - lens[b]].any()


@pytest.mark.parametrize("kscale,qscale", [(1e-4, 1.0), (30.0, 8.0), (1e3, 1e-2), (1e-20, 1e3), (1.0, 1e-30)])
def test_ranges_of_keys_and_queries(ip, kscale, qscale):
    q, ks, vs, cache, table = make(2, 1, 4, 2, [300, 77], 32, "bf16", seed=5, kscale=kscale, qscale=qscale)
    got = ip.kv4_attention(q, ints([300, 77]), table, cache, max_len=320)
    check(ip, got, q, ks, vs, [1, 1], True)


@pytest.mark.parametrize("lo,hi", [(-30, 30), (-100, -90), (90, 96)])
def test_ranges_of_values(ip, lo, hi):
    # values whose scale grows and shrinks by many powers of two along the sequence
    rng = np.random.default_rng(8)
    n = 500
    ks = [0.1 * rng.standard_normal((n, 1, 128))]
    vs = [rng.standard_normal((n, 1, 128)) * 2.0 ** rng.integers(lo, hi + 1, (n, 1, 1))]
    cache, table = ref.build_cache(ks, vs, 16, rng)
    q = torch.from_numpy(rng.standard_normal((1, 1, 2, 128))).to(torch.bfloat16).cuda()
    got = ip.kv4_attention(q, ints([n]), torch.from_numpy(table).cuda(), torch.from_numpy(cache).cuda(), max_len=n)
    check(ip, got, q, ks, vs, [1], True)


def test_not_finite_stays_in_its_place(ip):
    # a NaN in a cached key reaches the queries that see it; one in a value reaches its
    # group of channels; infinities behind a sequence's end reach nothing
    rng = np.random.default_rng(3)
    k, v = (torch.from_numpy(rng.standard_normal((2, 40, 2, 128))).float().cuda() for _ in range(2))
    k[0, 30, 0, 5] = float("nan")
    v[1, 10, 1, 70] = float("inf")
    cache = ip.kv4_cache(6, 2, 16)
    cache.fill_(255)
    table = ints([[0, 1, 2], [3, 4, 5]])
    ip.kv4_append(k, v, ints([0, 0]), table, cache)
    q = torch.randn(2, 3, 4, 128, device="cuda").to(torch.float16)
    # sequence 0: queries at positions 29, 30, 31; heads 0, 1 read cache head 0
    got = ip.kv4_attention(q, ints([32, 40]), table, cache)
    bad = torch.isnan(got)
    assert bad[0, 1:, :2].all() and not bad[0, 0].any() and not bad[0, :, 2:].any()
    assert bad[1, :, 2:, 64:96].all() and not bad[1, :, :2].any()
    assert not bad[1, :, 2:, :64].any() and not bad[1, :, 2:, 96:].any()


def test_the_other_groups_keep_their_values_beside_a_nan(ip):
    rng = np.random.default_rng(4)
    k, v = (torch.from_numpy(rng.standard_normal((1, 33, 1, 128))).float().cuda() for _ in range(2))
    cache, clean = ip.kv4_cache(3, 1, 16), ip.kv4_cache(3, 1, 16)
    table = ints([[2, 0, 1]])
    ip.kv4_append(k, v, ints([0]), table, clean)
    v2 = v.clone()
    v2[0, 20, 0, 64:96] = float("nan")
    ip.kv4_append(k, v2, ints([0]), table, cache)
    q = torch.randn(1, 1, 2, 128, device="cuda").to(torch.bfloat16)
    a, b = (ip.kv4_attention(q, ints([33]), table, c) for c in (clean, cache))
    keep = [i for i in range(128) if not 64 <= i < 96]
    assert torch.equal(a[..., keep], b[..., keep]) and torch.isnan(b[..., 64:96]).all()


def test_missing_pages_and_long_lengths_are_reported(ip):
    q, ks, vs, cache, table = make(2, 1, 2, 2, [100, 40], 16, "f16", seed=9)
    bad = table.clone()
    bad[0, 2] = -1
    bad[1, 1] = cache.shape[0]
    ws = space(ip.kv4_attention_workspace_bytes(2, 1, 2, 2, 100))
    got = ip.kv4_attention(q, ints([100, 40]), bad, cache, max_len=100, workspace=ws)
    assert ip.status(ws) == -7
    cut = [np.concatenate([x[0][:32], x[0][48:]]) for x in (ks, vs)], [np.concatenate([x[1][:16], x[1][32:]])
                                                                     for x in (ks, vs)]
    check(ip, got, q, [cut[0][0], cut[1][0]], [cut[0][1], cut[1][1]], [1, 1], False)
    got = ip.kv4_attention(q, ints([100, 40]), table, cache, max_len=64, workspace=ws)
    assert ip.status(ws) == -7
    check(ip, got, q, [ks[0][:64], ks[1]], [vs[0][:64], vs[1]], [1, 1], False)
    got = ip.kv4_attention(q, ints([-5, 40]), table, cache, max_len=64, workspace=ws)
    assert ip.status(ws) == 0 and not got[0].any()


def test_strided_queries_other_stream_and_graph(ip):
    q, ks, vs, cache, table = make(3, 2, 8, 2, [70, 200, 33], 16, "bf16", seed=11)
    lens = ints([70, 200, 33])
    size = ip.kv4_attention_workspace_bytes(3, 2, 8, 2, 256)
    ws = space(size)
    base = torch.randn(3, 2, 3 * 1024 + 3, device="cuda").to(torch.bfloat16)
    view = base[..., 3:1027].unflatten(-1, (8, 128))
    view.copy_(q)
    call = lambda x, **kw: ip.kv4_attention(x, lens, table, cache, max_len=200, workspace=ws, **kw)
    want = call(q)
    assert torch.equal(call(view), want)
    assert torch.equal(call(q.transpose(1, 2).contiguous().transpose(1, 2)), want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(q, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    ws.fill_(255)      # but for its status word the workspace may hold anything
    ws[:256] = 0
    assert torch.equal(call(q), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(q)
    for n in ([70, 200, 33], [1, 0, 30], [64, 65, 16]):
        lens.copy_(ints(n))
        graph.replay()
        torch.cuda.synchronize()
        check(ip, out, q, [x[:i] for x, i in zip(ks, n)], [x[:i] for x, i in zip(vs, n)], [2] * 3, True)
    assert ip.status(ws) == 0


def test_decode_steps_end_to_end(ip):
    """A prompt and single tokens through product, cache and attention as a decoder's layer
    has them, each step against float64 on the values that the cache holds."""
    B, H, Hkv, D = 2, 8, 2, 256
    g = torch.Generator(device="cuda").manual_seed(12)
    N = (H + 2 * Hkv) * 128
    wq, sw = ip.quantize_rows_i8(torch.randn(N, D, generator=g, device="cuda") / 16)
    wo, so = ip.quantize_rows_i8(torch.randn(D, H * 128, generator=g, device="cuda") / 32)
    cache, table = ip.kv4_cache(9, Hkv, 16), ints([[3, 1, 7], [0, 8, 2]])
    ws = space(ip.kv4_attention_workspace_bytes(B, 20, H, Hkv, 48))
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    ks, vs = [np.zeros((0, Hkv, 128))] * B, [np.zeros((0, Hkv, 128))] * B
    for T, counts in ((20, [20, 11]), (1, [1, 1]), (1, [1, 0]), (3, [2, 3])):
        x = torch.randn(B, T, D, generator=g, device="cuda").to(torch.bfloat16)
        cnt = ints(counts)
        xq, sx = ip.quantize_rows_i8(x)
        qkv = ip.linear_scaled_i8(xq, sx, wq, sw, dtype=torch.bfloat16, workspace=ws)
        heads = qkv.unflatten(-1, (H + 2 * Hkv, 128))
        q, k, v = heads[:, :, :H], heads[:, :, H:H + Hkv], heads[:, :, H + Hkv:]
        ip.kv4_append(k, v, lens, table, cache, count=cnt, workspace=ws)
        lens = lens + cnt
        o = ip.kv4_attention(q, lens, table, cache, count=cnt, max_len=48, workspace=ws)
        oq, s = ip.quantize_rows_i8(o.flatten(2))
        y = ip.linear_scaled_i8(oq, s, wo, so, dtype=torch.float32, workspace=ws)
        for b in range(B):
            ks[b] = np.concatenate([ks[b], f64(k)[b, :counts[b]]])
            vs[b] = np.concatenate([vs[b], f64(v)[b, :counts[b]]])
        check(ip, o, q, ks, vs, counts, True)
        want = (oq.double() @ wo.double().t()) * s.double()[..., None] * so.double()
        assert (y.double() - want).abs().max() <= want.abs().max() * 2.0 ** -22
    assert ip.status(ws) == 0
