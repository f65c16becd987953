"""The attention over the 4-bit cache at the ends of the scores' range: queries next to the
largest bf16 number, scores that f32 holds in steps of more than one, query rows of zeros."""
import numpy as np
import pytest

import kv4_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ip():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_30846_gb300 as ip
    ip.load()
    return ip


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def cached(ks, vs, page, seed):
    cache, table = ref.build_cache(ks, vs, page, np.random.default_rng(seed))
    return torch.from_numpy(cache).cuda(), torch.from_numpy(table).cuda()


@pytest.mark.parametrize("exponent", [100, 120, 121, 122, 125])
@pytest.mark.parametrize("n,T,H", [(5, 1, 2), (300, 1, 4), (900, 3, 8)])
def test_queries_next_to_the_largest_number(ip, exponent, n, T, H):
    # one key lies along the query, the others are a hundredth of it: all weight is that token's,
    # whose value is c s, exact but for the rounding of the output.  |q| 2^exponent on sixteen channels
    # keeps q k below 2^(exponent + 2)
    rng = np.random.default_rng(n + exponent)
    sign = np.where(rng.random(16) < 0.5, -1.0, 1.0)
    k, v = 0.0025 * rng.uniform(-1, 1, (n, 1, 128)), rng.standard_normal((n, 1, 128))
    best = n // 3
    k[best, 0, ::8] = 0.25 * sign
    q = np.zeros((1, T, H, 128))
    q[..., ::8] = sign * 2.0 ** exponent * (1 + np.arange(H)[:, None] / 8)
    cache, table = cached([k], [v], 16, 1)
    got = ip.kv4_attention(torch.from_numpy(q).to(torch.bfloat16).cuda(), ints([n]), table, cache, causal=False)
    want = torch.from_numpy(ref.values(v)[best, 0]).to(torch.bfloat16).cuda()
    assert torch.equal(got, want.expand_as(got))


@pytest.mark.parametrize("scale", [None, 1e-30, 1e20])
def test_keys_of_zeros_under_large_queries(ip, scale):
    # scores of 0 for every third token and far below for the others: the mean of those tokens
    n, exponent = 400, {None: 124, 1e-30: 125, 1e20: 40}[scale]
    rng = np.random.default_rng(3)
    k, v = np.zeros((n, 1, 128)), rng.standard_normal((n, 1, 128))
    q = np.full((1, 1, 8, 128), 2.0 ** exponent)
    k[1::3] = k[2::3] = -0.01
    cache, table = cached([k], [v], 64, 2)
    got = ip.kv4_attention(torch.from_numpy(q).to(torch.bfloat16).cuda(), ints([n]), table, cache, scale=scale)
    x = ref.values(v)[::3, 0]
    want, mag = x.mean(0), np.abs(x).mean(0)
    # p s to fp16 (2^-11), the f32 sums, the output to bf16 (2^-8)
    tol = mag * (2.0 ** -11 + 2.0 ** -16) * 1.01 + np.abs(want) * 2.0 ** -8
    assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("T,n", [(6, 6), (20, 40), (33, 700)])
@pytest.mark.parametrize("scale", [1e-8, 1e-12, None])
def test_query_rows_of_zeros(ip, page, T, n, scale):
    # equal scores: the mean of the values that each row sees, beside rows with large scores
    rng = np.random.default_rng(T)
    k, v = rng.standard_normal((n, 1, 128)), rng.standard_normal((n, 1, 128))
    q = rng.standard_normal((1, T, 2, 128)) * 1e9
    q[:, ::2] = 0
    cache, table = cached([k], [v], page, 3)
    got = ip.kv4_attention(torch.from_numpy(q).to(torch.bfloat16).cuda(), ints([n]), table, cache, scale=scale,
                           max_len=n).double().cpu().numpy()
    x = ref.values(v)[:, 0]
    top = np.abs(x).max() / 7 * 1.01
    assert np.isfinite(got).all()
    for t in range(0, T, 2):
        seen = x[:n - T + t + 1]
        want, mag = seen.mean(0), np.abs(seen).mean(0)
        tol = mag * (2.0 ** -11 + 2.0 ** -16) * 1.01 + np.abs(want) * 2.0 ** -8 + n * 2.0 ** -34 * 7 * top
        assert (np.abs(got[0, t] - want) <= tol).all()
