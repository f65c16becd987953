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


@pytest.mark.parametrize("what", ["nan", "inf", "huge"])
@pytest.mark.parametrize("T,H,page", [(4, 2, 16), (7, 1, 32), (40, 2, 64)])
def test_what_a_query_does_not_see_does_not_reach_it(ip, what, T, H, page):
    # causal queries before the tokens that hold a NaN, infinities or values 2^60 times the others':
    # the definition's output, as if the later tokens were not there
    n, bad = 90 + T, T // 2          # the queries at 90 + bad and later see them
    q, ks, vs, _, _ = make(1, T, H, 1, [n], page, "bf16", seed=T)
    val = {"nan": float("nan"), "inf": float("-inf"), "huge": 2.0 ** 60}[what]
    for x in (ks, vs) if what != "huge" else (vs,):
        x[0][90 + bad:, 0, 70::9] = val
    cache = ip.kv4_cache(-(-n // page), 1, page)
    table = ints([list(range(-(-n // page)))[::-1]])
    k, v = (torch.from_numpy(x[0][None]).float().cuda() for x in (ks, vs))
    ip.kv4_append(k, v, ints([0]), table, cache)
    got = ip.kv4_attention(q, ints([n]), table, cache, max_len=n)
    m = 90 + bad
    cut = [[f64(x)[0, :m]] for x in (k, v)]
    check(ip, got[:, :bad], q[:, :bad], *cut, [bad], True)
    if what != "huge":
        assert torch.isnan(got[:, bad:]).all()
        only_v = ip.kv4_cache(-(-n // page), 1, page)
        ip.kv4_append(torch.nan_to_num(k, 1.0, 1.0, -1.0), v, ints([0]), table, only_v)
        got = torch.isnan(ip.kv4_attention(q, ints([n]), table, only_v, max_len=n))
        assert got[:, bad:, :, 64:].all() and not got[:, bad:, :, :64].any() and not got[:, :bad].any()


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


# ------------------------------------------------------------ larger shapes, on the GPU's own values

def big_check(ip, B, T, H, Hkv, lens, counts, page, dtype, causal, seed, scale=None, max_len=None, heads_off=0):
    """Attention against float64 torch on the values that kv4_read gives (pinned above), with
    kv4_ref.attention's bound."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-n // page) for n in lens]
    total = sum(need) + 2
    ids = torch.randperm(total, generator=g, device="cuda").int()
    table = torch.full((B, max(1, max(need))), -7, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    cache = ip.kv4_cache(total, Hkv, page)
    cache.fill_(255)
    L = max(1, max(lens))
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    ws = space(ip.kv4_attention_workspace_bytes(B, T, H, Hkv, max(L, max_len or 0)))
    for b in range(B):      # one sequence at a time bounds the memory
        if lens[b]:
            k, v = (torch.randn(1, lens[b], Hkv, 128, generator=g, device="cuda") for _ in range(2))
            ip.kv4_append(k, v, zero[:1], table[b:b + 1], cache, workspace=ws)
    q = (1.5 * torch.randn(B, T, H, 128, generator=g, device="cuda")).to(DT[dtype])
    cnt = None if counts is None else ints(counts)
    out = ip.kv4_attention(q, ints(lens), table, cache, count=cnt, causal=causal, scale=scale,
                           max_len=max_len, workspace=ws if max_len else None)
    assert ip.status(ws) == 0
    sc = 128 ** -0.5 if scale is None else scale
    eps = torch.finfo(q.dtype).eps
    for b in range(B):
        c = T if counts is None else min(counts[b], T)
        assert not out[b, c:].any()
        n = lens[b]
        if n == 0 or c == 0:
            assert not out[b].any()
            continue
        k, v = ip.kv4_read(cache, zero[:1], table[b:b + 1], n, dtype=torch.float32)
        k, v = (x[0].double().repeat_interleave(H // Hkv, 1).transpose(0, 1) for x in (k, v))      # [H, n, 128]
        qq = q[b, :c].double().transpose(0, 1)
        x = qq @ k.transpose(1, 2) * sc
        if causal:
            x = x.masked_fill(torch.arange(n, device="cuda") > n - c + torch.arange(c, device="cuda")[:, None], -np.inf)
        p = torch.nan_to_num(torch.softmax(x, -1))
        want = p @ v
        # 15 s sum |q| <= 15 max(s) sum |q|, s <= max|k| / 7 (1 + 2^-8) in a group
        A = 15 / 7 * 1.01 * k.abs().amax((1, 2), keepdim=True) * qq.abs().sum(-1, keepdim=True) * sc
        rel = 2 * 2.0 ** -20 * A + 2.0 ** -11 + 2.0 ** -16 + n * 2.0 ** -28
        top = v.abs().amax((1, 2), keepdim=True) * 1.01
        tol = rel * (p @ v.abs()) + n * 2.0 ** -34 * top
        # a result below the type's normal range rounds by half of smallest_normal eps (2^-25 for f16)
        tol = tol * (1 + eps) + want.abs() * eps / 2 + torch.finfo(q.dtype).smallest_normal * eps
        err = (out[b, :c].double().transpose(0, 1) - want).abs()
        assert (err <= tol).all(), (b, float((err / tol).max()))


@pytest.mark.parametrize("case", [
    dict(B=2, T=1, H=8, Hkv=2, lens=[70001, 333], page=32, causal=True),            # one long, one short
    dict(B=40, T=1, H=8, Hkv=4, lens=[(37 * i * i) % 900 for i in range(40)], page=16, causal=True),
    dict(B=1, T=700, H=4, Hkv=2, lens=[1100], page=64, causal=True),                # a long chunk
    dict(B=2, T=300, H=3, Hkv=3, lens=[300, 37], page=16, causal=False),
    dict(B=2100, T=1, H=2, Hkv=1, lens=[(i * 7) % 200 for i in range(2100)], page=16, causal=True),   # a CTA an item
    dict(B=3, T=2, H=96, Hkv=2, lens=[500, 20, 1], page=16, causal=True),           # 48 heads to a cache head
], ids=["long", "ragged", "chunk", "cross", "items", "groups"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_at_size(ip, case, dtype):
    big_check(ip, counts=None, dtype=dtype, seed=len(case["lens"]), **case)


def test_attention_seeded_sweep(ip):
    rng = np.random.default_rng(5)
    for i in range(40):
        B, Hkv, G = int(rng.integers(1, 12)), int(rng.choice([1, 2, 3, 8])), int(rng.choice([1, 2, 4, 7]))
        T = int(rng.choice([1, 1, 2, 5, 17, 40]))
        top = int(np.exp(rng.uniform(0, np.log(5000))))
        lens = [int(x) for x in rng.integers(0, top + 1, B)]
        counts = None if rng.random() < 0.5 else [int(x) for x in rng.integers(0, T + 2, B)]
        big_check(ip, B, T, G * Hkv, Hkv, lens, counts, int(rng.choice([16, 32, 64])), ["f16", "bf16"][i % 2],
                  bool(rng.random() < 0.6), seed=i, scale=None if rng.random() < 0.5 else float(rng.uniform(0.01, 0.3)),
                  max_len=None if rng.random() < 0.5 else top + int(rng.integers(1, 4000)))


def test_a_cache_past_31_bits(ip):
    H, page = 8, 64
    n_pages = (5 << 30) // (H * 144 * page)
    cache = torch.empty(n_pages, H, 144 * page, dtype=torch.uint8, device="cuda")
    small = ip.kv4_cache(4, H, page)
    far, near = ints([[n_pages - 1, n_pages // 2 + 3, n_pages - 7]]), ints([[2, 0, 3]])
    k, v = (torch.randn(1, 170, H, 128, device="cuda") for _ in range(2))
    q = torch.randn(1, 1, H, 128, device="cuda").half()
    res = []
    for c, t in ((cache, far), (small, near)):
        ip.kv4_append(k, v, ints([0]), t, c)
        res.append((ip.kv4_attention(q, ints([170]), t, c), *ip.kv4_read(c, ints([0]), t, 170)))
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_refusals(ip):
    q = torch.zeros(2, 1, 4, 128, device="cuda").half()
    k = torch.zeros(2, 3, 2, 128, device="cuda").half()
    cache, table, i2 = ip.kv4_cache(4, 2, 16), ints([[0], [1]]), ints([0, 1])
    ok = dict(q=q, lengths=i2, page_table=table, cache=cache)
    ip.kv4_attention(**ok)
    for err, over in ((TypeError, dict(q=q.float())), (TypeError, dict(lengths=i2.long())), (TypeError, dict(lengths=None)),
                      (ValueError, dict(lengths=ints([1]))), (ValueError, dict(count=ints([1]))),
                      (ValueError, dict(page_table=ints([[0]]))), (TypeError, dict(page_table=table.cpu())),
                      (ValueError, dict(cache=cache[:, :, :-1])), (TypeError, dict(cache=cache.to(torch.int8))),
                      (ValueError, dict(q=q[..., ::2])), (ValueError, dict(q=q.transpose(2, 3))),
                      (ip.IpError, dict(q=torch.zeros(2, 1, 3, 128, device="cuda").half())),
                      (ip.IpError, dict(scale=-1.0)), (ip.IpError, dict(max_len=-1)),
                      (ip.IpError, dict(q=torch.zeros(2, 0, 4, 128, device="cuda").half())),
                      (ip.IpError, dict(q=torch.zeros(2, 2049, 4, 128, device="cuda").half())),
                      (ip.IpError, dict(cache=torch.zeros(4, 2, 144 * 8, dtype=torch.uint8, device="cuda"))),
                      (ip.IpError, dict(workspace=torch.zeros(300, dtype=torch.uint8, device="cuda"), max_len=4096))):
        with pytest.raises(err):
            ip.kv4_attention(**dict(ok, **over))
    ok = dict(k=k, v=k, start=i2, page_table=table, cache=cache)
    ip.kv4_append(**ok)
    for err, over in ((ValueError, dict(v=k[:, :2])), (TypeError, dict(v=k.float())), (TypeError, dict(start=None)),
                      (ValueError, dict(k=k[:, :, :1], v=k[:, :, :1])), (TypeError, dict(k=k.int(), v=k.int())),
                      (ValueError, dict(k=k[..., :64], v=k[..., :64])),
                      (ValueError, dict(k=k.transpose(2, 3).contiguous().transpose(2, 3)))):
        with pytest.raises(err):
            ip.kv4_append(**dict(ok, **over))
    with pytest.raises(TypeError):
        ip.kv4_read(cache, i2, table, 2, dtype=torch.float64)
    with pytest.raises(ValueError):
        ip.kv4_read(cache, i2, table, -1)


def test_append_where_the_scale_is_subnormal(ip):
    # the nearest scale may be a third below amax / 7: codes end at 7
    unit = 2.0 ** -133                      # of a bf16 subnormal
    rng = np.random.default_rng(12)
    x = np.zeros((1, 64, 1, 128), np.float32)
    for t in range(64):
        x[0, t, 0] = (rng.uniform(-1, 1, 128) * unit * rng.uniform(1, 60)).astype(np.float32)
        x[0, t, 0, 32 * (t % 4)] = np.float32(unit * (3.6 + 0.17 * t))
    k = torch.from_numpy(x).cuda()
    cache, table = ip.kv4_cache(1, 1, 64), ints([[0]])
    ip.kv4_append(k, -k, ints([0]), table, cache)
    got = cache.cpu().numpy()[0, 0]
    base = 0
    for part, size in zip((*ref.rows_bytes(f64(k)[0, :, 0], ref.K_BYTE), *ref.rows_bytes(f64(-k)[0, :, 0], ref.V_BYTE)),
                          (64, 8, 64, 8)):
        np.testing.assert_array_equal(got[base:base + 64 * size].reshape(64, size), part)
        base += size * 64
