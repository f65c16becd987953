"""Zeros that kv4_read writes are positive, bit for bit: rows past the count, positions without a
page, channels whose code is 0."""
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


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_zeros_read_back_are_positive(ip, dtype):
    cache, table = ip.kv4_cache(3, 2, 16), ints([[0, -1], [2, 1]])
    x = torch.randn(2, 20, 2, 128, device="cuda")
    x[1, 3, 1, 32:64] = 0
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    ip.kv4_append(x, x, ints([0, 0]), table, cache, count=ints([16, 20]), workspace=ws)
    assert ip.status(ws) == 0
    bits = torch.int32 if dtype == torch.float32 else torch.int16
    # sequence 0: its second page does not exist; 1: rows past the count
    for t in ip.kv4_read(cache, ints([0, 0]), table, 20, count=ints([20, 9]), dtype=dtype, workspace=ws):
        assert not t[0, 16:].contiguous().view(bits).any() and not t[1, 9:].contiguous().view(bits).any()
        assert not t[1, 3, 1, 32:64].contiguous().view(bits).any()
        assert t[0, :16].any() and t[1, :9].any()
    assert ip.status(ws) == -7
