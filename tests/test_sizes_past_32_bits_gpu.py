"""Sizes and choices that 32 bits do not hold, through the calls on tensors: refused, not wrapped."""
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


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_arguments_outside_32_bits(ip):
    q = torch.randn(2, 1, 4, 128, device="cuda").half()
    cache, table, lens = ip.kv4_cache(4, 2, 16), ints([[0], [1]]), ints([3, 16])
    ws = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    for space in (None, ws):
        for n in (2 ** 32 + 1, 2 ** 32, 2 ** 31, -2 ** 32 + 5, 2 ** 70):
            with pytest.raises(ip.IpError):
                ip.kv4_attention(q, lens, table, cache, max_len=n, workspace=space)
    x, w = torch.zeros(2, 32, dtype=torch.int8, device="cuda"), torch.zeros(5, 32, dtype=torch.int8, device="cuda")
    for space in (None, ws):
        for act in (2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 70):
            with pytest.raises(ip.IpError):
                ip.linear_scaled_i8(x, torch.ones(2, device="cuda"), w, torch.ones(5, device="cuda"), act=act,
                                    workspace=space)


def test_sizes_of_expanded_tensors(ip):
    # 2^32 + 1 tokens without memory of their own
    k = torch.zeros(1, 1, 2, 128, device="cuda").half().expand(1, 2 ** 32 + 1, 2, 128)
    cache, table, start = ip.kv4_cache(4, 2, 16), ints([[0, 1]]), ints([0])
    before = cache.clone()
    for space in (None, torch.zeros(256, dtype=torch.uint8, device="cuda")):
        with pytest.raises(ip.IpError):
            ip.kv4_append(k, k, start, table, cache, workspace=space)
    assert torch.equal(cache, before)
