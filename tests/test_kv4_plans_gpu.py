"""The attention over the 4-bit cache where its items or units are too many to be dealt in shares."""
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


def test_a_bound_of_the_lengths_far_above_them(ip):
    # 64 sequences, 2048 queries, a bound of 2^20 and of 2^28: as with a close one
    B, T, H, Hkv, page, n = 64, 2048, 4, 2, 16, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    cache, ids = ip.kv4_cache(3 * B, Hkv, page), torch.randperm(3 * B, generator=g, device="cuda").int().view(B, 3)
    k, v = (torch.randn(B, n, Hkv, 128, generator=g, device="cuda") for _ in range(2))
    lens = torch.randint(0, n + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    table = torch.zeros(B, 1 << 16, dtype=torch.int32, device="cuda")
    table[:, :3] = ids
    ip.kv4_append(k, v, torch.zeros_like(lens), table, cache)
    q = torch.randn(B, 1, H, 128, generator=g, device="cuda").half().expand(B, T, H, 128)
    want = ip.kv4_attention(q, lens, table, cache, causal=False, max_len=n)
    for bound in (None, 1 << 20, 1 << 28):
        assert torch.equal(ip.kv4_attention(q, lens, table, cache, causal=False, max_len=bound), want)


def test_more_than_2_24_rows_of_a_cache_head(ip):
    T, H, n = 2048, 8200, 3
    rng = np.random.default_rng(2)
    ks, vs = [rng.standard_normal((n, 1, 128))], [rng.standard_normal((n, 1, 128))]
    cache, table = ref.build_cache(ks, vs, 16, rng)
    q = torch.randn(1, 1, 1, 128, device="cuda").half()
    args = ints([n]), torch.from_numpy(table).cuda(), torch.from_numpy(cache).cuda()
    want = ip.kv4_attention(q, *args, causal=False, max_len=n)
    got = ip.kv4_attention(q.expand(1, T, H, 128), *args, causal=False, max_len=n)
    assert got.numel() > 2 ** 31 and torch.equal(got, want.expand_as(got))
