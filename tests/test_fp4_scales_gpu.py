"""Every block scale that the product of 4-bit rows reads, in each of its forms (few rows by ordinary lanes, tiles,
tiles whose K a cluster shares, tiles of a pair of CTAs): exactly what float64 gives."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import fp4_ref as ref


@pytest.fixture(scope="module")
def ip():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_30846_gb300 as ip
    ip.load()
    return ip


def rows(n, K, seed, one_block, first=0):
    """Random codes, row i with block scales of byte (first + i) mod 127 (all there are from 0 on but NaN).  one_block: codes in
    block i mod K / 16 alone, so that a product is one block's: two scales of four bits and a sum of codes, exact in f32."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.randint(0, 16, (n, K), generator=g, device="cuda", dtype=torch.uint8)
    i = torch.arange(n, device="cuda")
    if one_block:
        c = torch.where((torch.arange(K, device="cuda") // 16)[None] == (i % (K // 16))[:, None], c, 0)
    q, blocks = ref.bytes_of(c, ((first + i) % 127).to(torch.uint8)[:, None].expand(n, K // 16))
    return q, blocks, torch.ones(n, device="cuda")


def check(ip, x, w, K):
    want = ref.values(*x, K) @ ref.values(*w, K).t()
    y = ip.linear_fp4(*x, *w, dtype=torch.float32)
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("M", [1, 2, 4, 8])
def test_few_rows(ip, M):
    w = rows(127, 320, 1, False)
    for first in range(0, 127, M):
        check(ip, rows(M, 320, first, True, first), w, 320)


@pytest.mark.parametrize("M,K,N", [(127, 320, 127), (127, 4096, 127), (300, 1024, 1000), (4096, 1024, 4096)])
def test_tiles(ip, M, K, N):
    check(ip, rows(M, K, 3, True), rows(N, K, 4, False), K)
