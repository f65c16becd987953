"""The scaled product's bounded waits: with the stall hook the output warps wait on a barrier that
nothing arrives on, the limit of about a millisecond runs out, every role gives up (copies in
flight land, MMAs end, TMEM is freed), the status word says so, and the next call is exact."""
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


# one CTA a tile of 32 channels, K in two and in four parts, tiles of 128 x 128 and pairs, with one
# segment of K and several, fewer tiles than SMs and more, rows of any alignment
SIZES = [(200, 1024, 1000), (512, 900, 512), (200, 4096, 1000), (128, 4096, 512), (128, 8192, 500), (150, 64, 24576),
         (130, 2500, 9000), (2000, 3000, 5001), (40, 700, 4097), (600, 5000, 4096), (3000, 1024, 4096), (3000, 3000, 8193)]


@pytest.mark.parametrize("M,K,N", SIZES)
def test_every_role_gives_up_and_the_next_call_is_exact(ip, M, K, N):
    g = torch.Generator(device="cuda").manual_seed(M)
    ld = -(-K // 16) * 16
    x, w = (torch.randint(-128, 128, (n, ld), generator=g, device="cuda", dtype=torch.int8)[:, :K] for n in (M, N))
    ones = torch.ones(max(M, N), device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    want = (x.double() @ w.double().t()).float()
    call = lambda: ip.linear_scaled_i8(x, ones[:M], w, ones[:N], dtype=torch.float32, workspace=ws)
    assert torch.equal(call(), want) and ip.status(ws) == 0
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


def test_few_tokens_wait_for_nothing(ip):
    x = torch.ones(1, 64, dtype=torch.int8, device="cuda")
    w, ws = torch.ones(48, 64, dtype=torch.int8, device="cuda"), torch.zeros(256, dtype=torch.uint8, device="cuda")
    try:
        ip.set_timeout_cycles(2_000_000)
        ip.set_stall_injection(True)
        y = ip.linear_scaled_i8(x, torch.ones(1, device="cuda"), w, torch.ones(48, device="cuda"), workspace=ws)
        assert (y == 64).all() and ip.status(ws) == 0
    finally:
        ip.set_stall_injection(False)
        ip.set_timeout_cycles(-1)
