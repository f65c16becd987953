"""The native short forms leave what is not theirs to the general forms (no GPU needed)."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ip():
    import paper_2609_30846_gb300 as ip
    ip.load()
    if ip._short is ip._Unbound:
        pytest.skip("no torch with CUDA to build for")
    return ip


X = torch.zeros(2, 16, dtype=torch.int8)
F = torch.zeros(2, 16)
JUNK = (None, 3, "x", 1.5, [1], object(), X, F, F[0, 0], torch.zeros(0), torch.float32)


@pytest.mark.parametrize("name,n", [("quantize_rows", 3), ("linear_scaled", 9), ("kv4_append", 7), ("kv4_read", 7),
                                    ("kv4_attention", 10)])
def test_nothing_but_plain_cuda_tensors_is_taken(ip, name, n):
    f = getattr(ip._short, name)
    for j in JUNK:
        assert f(*[j] * n) is None
    for i in range(n):
        assert f(*[F if k != i else None for k in range(n)]) is None
    for m in (0, n - 1, n + 1):
        with pytest.raises(TypeError):
            f(*[None] * m)


def test_the_general_forms_name_what_is_wrong(ip):
    for call in (lambda: ip.quantize_rows_i8(F), lambda: ip.quantize_rows_i8(None),
                 lambda: ip.linear_scaled_i8(X, F[:, 0], X, F[:, 0]),
                 lambda: ip.kv4_append(F, F, None, None, None), lambda: ip.kv4_read(F, F, F, 1),
                 lambda: ip.kv4_attention(F, F, F, F)):
        with pytest.raises(TypeError, match="CUDA tensor"):
            call()


def test_bind_wants_the_entry_points(ip):
    with pytest.raises(TypeError):
        ip._short.bind(1, 2)
    with pytest.raises(TypeError):
        ip._short.bind("a", 2, 3, 4, 5)
