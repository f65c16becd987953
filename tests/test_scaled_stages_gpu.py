"""The scaled product where every stage of the pipeline is another tile's (K up to 64) and where
tiles change in the middle of the ring: bit for bit the exact integers, again and again."""
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


@pytest.mark.parametrize("M,N", [(150, 24576), (3000, 1536), (20000, 2048), (9000, 4100), (257, 30000)])
@pytest.mark.parametrize("K", [16, 33, 64, 65, 200, 320, 450, 1100])
def test_products_repeat_and_are_exact(ip, M, N, K):
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    ld = -(-K // 16) * 16
    x, w = (torch.randint(-128, 128, (n, ld), generator=g, device="cuda", dtype=torch.int8)[:, :K] for n in (M, N))
    one = lambda n: torch.ones(n, device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    want = x.double() @ w.double().t()
    want = want.float()                    # |sums| < 2^25 in 64 bits: one rounding
    flush = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    for i in range(6):
        if i % 2:
            flush.fill_(i)                 # every copy from DRAM
        y = ip.linear_scaled_i8(x, one(M), w, one(N), dtype=torch.float32, workspace=ws)
        assert torch.equal(y, want)
    assert ip.status(ws) == 0
