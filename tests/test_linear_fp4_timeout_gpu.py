"""The 4-bit product's bounded waits: with the stall hook the output warps wait on a barrier that
nothing arrives on, the limit of about a millisecond runs out, every role gives up (copies in flight
land, MMAs end, TMEM is freed), the status word says so, and the next call is right."""
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


# tiles of 128 x 64, of 128 x 128 and of 256 x 256 by two CTAs; one stage and more than the buffers hold, one
# tile an SM and several, output rows of any alignment
SIZES = [(9, 100, 64), (13, 1024, 1000), (40, 4096, 300), (200, 20000, 1000), (128, 8192, 512), (300, 256, 4096), (300, 3000, 4097), (1500, 1024, 4096), (4096, 1024, 4096),
         (3000, 8192, 4096), (2049, 200, 8193)]


@pytest.mark.parametrize("M,K,N", SIZES)
def test_every_role_gives_up_and_the_next_call_is_right(ip, M, K, N):
    g = torch.Generator(device="cuda").manual_seed(M)
    x = ip.quantize_fp4(torch.randn(M, K, generator=g, device="cuda"))
    w = ip.quantize_fp4(torch.randn(N, K, generator=g, device="cuda"))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    call = lambda: ip.linear_fp4(*x, *w, workspace=ws)
    want = call()
    assert ip.status(ws) == 0
    for _ in range(3):
        try:
            ip.set_timeout_cycles(2_000_000)
            ip.set_stall_injection(True)
            call()
            assert ip.status(ws) == -6          # IP_ERR_TIMEOUT, read and cleared
            assert ip.status(ws) == 0
        finally:
            ip.set_stall_injection(False)
            ip.set_timeout_cycles(-1)
        assert torch.equal(call(), want) and ip.status(ws) == 0
