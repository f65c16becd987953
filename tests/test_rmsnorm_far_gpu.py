"""The norm at the top of the range without eps: the factor 1 / root lies below the normal numbers there, the scale does not."""
import pytest

from test_rmsnorm_gpu import DT, check, draw, ip  # noqa: F401 - a fixture

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e37, 1e38, 3e38])
@pytest.mark.parametrize("d", [1, 17, 300, 2000, 9000, 32768])
def test_largest_rows_without_eps(ip, dtype, scale, d):  # noqa: F811
    x, g, _ = draw(5, d, torch.float32, d, False)
    x = (x / x.abs().amax(1, keepdim=True) * scale).to(DT[dtype])
    g = (g / g.abs().amax()).to(DT[dtype])
    x[1] = 0
    x[2, 1:] = 0
    x[3] = scale                      # the largest root: all elements as far out
    check(ip, x, g, eps=0.0)
    check(ip, x, g, eps=1e-5)
