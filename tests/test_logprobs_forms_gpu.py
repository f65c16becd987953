"""Rows of logits at the ends of the warp's forms, on 16 bytes and off."""
import pytest

from test_logprobs_gpu import check, ip  # noqa: F401 - a fixture

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("V", [248, 249, 264, 280, 281, 504, 505, 520, 536, 537, 1016, 1017, 1032, 1048, 1049])
def test_ends(ip, dtype, V):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(V)
    base = (4 * torch.randn(7, V + 8, generator=g, device="cuda")).to(dtype)
    for at in range(8):
        x = base[:, at:at + V]
        x[0, V - 1], x[1, 0], x[2, V // 2] = 30.0, 31.0, 32.0
        x[3, :V - 2] = -float("inf")                 # what is left lies in the elements more
        x[4] = 0.5
        tok = torch.tensor([V - 1, 0, V // 2, V - 2, V - 1, 1, V - 3], device="cuda", dtype=torch.int32)
        for top in (0, 1, 9, 32):
            check(ip, x, tok, top)
