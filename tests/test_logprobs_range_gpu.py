"""Log probabilities of logits that are further apart than f32 reaches: differences that overflow before
`scale` brings them back."""
import pytest

from test_logprobs_gpu import check, ip  # noqa: F401 - a fixture

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
# a warp's row, a CTA's, a cluster's, and one of parts that a second kernel joins
@pytest.mark.parametrize("V", [2, 40, 1025, 5000, 40000, 300000])
def test_differences_past_f32(ip, dtype, V):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(V)
    x = ((torch.rand(6, V, generator=g, device="cuda") * 2 - 1) * 3e38).to(dtype)
    x[:, 0], x[:, V - 1] = 3.2e38, -3.2e38
    x[1] = -x[1]
    x[2, 1:] = -3.2e38                  # all the weight on one, the others as far as can be
    x[3, :-1] = 3.2e38
    x[4, V // 2] = -float("inf")
    tok = torch.tensor([V - 1, 0, V - 1, V - 1, V // 2, V // 3], device="cuda", dtype=torch.int32)
    # powers of two, which f32 holds as they are (2^-130 as a subnormal number)
    for scale in (2.0 ** -130, 2.0 ** -126, 2.0 ** -125, 2.0 ** -120, 2.0 ** -60, 2.0 ** -3):
        check(ip, x, tok, min(V, 9), scale=scale)
        check(ip, x, tok.flip(0), min(V, 32), scale=scale)
