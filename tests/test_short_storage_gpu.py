"""Small new outputs of a call share one storage, as the calls' documents say: they do not overlap, and copies
stand alone."""
import copy
import io

import pytest

from test_short_forms_gpu import ip  # noqa: F401 - a fixture

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def outputs(ip, rows, d):  # noqa: F811
    x = torch.randn(rows, d, device="cuda").bfloat16()
    g, tok = torch.ones(d, device="cuda").bfloat16(), torch.zeros(rows, dtype=torch.int32, device="cuda")
    ws = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    return {"quantize_fp4": lambda: ip.quantize_fp4(x), "rmsnorm_i8": lambda: ip.rmsnorm_i8(x, g, x),
            "rmsnorm_fp4": lambda: ip.rmsnorm_fp4(x, g, x),
            "token_logprobs": lambda: ip.token_logprobs(x, tok, top=3, workspace=ws)}


@pytest.mark.parametrize("rows,d", [(1, 33), (5, 100), (130, 1000)])
def test_outputs_lie_apart(ip, rows, d):  # noqa: F811
    for name, call in outputs(ip, rows, d).items():
        out = call()
        keep = [t.clone() for t in out]
        for i, t in enumerate(out):
            t.zero_()
            for j, o in enumerate(out):
                if i != j:
                    assert torch.equal(o, keep[j]) or j < i, name
            if i:
                assert not out[i - 1].any(), name


def test_copies_stand_alone(ip):  # noqa: F811
    for name, call in outputs(ip, 5, 100).items():
        out = call()
        for t in out:
            c, d, f = t.clone(), copy.deepcopy(t), io.BytesIO()
            assert c.untyped_storage().data_ptr() != t.untyped_storage().data_ptr()
            c.untyped_storage().resize_(0)
            torch.save(t, f)
            f.seek(0)
            assert torch.equal(torch.load(f), t) and torch.equal(d, t), name


def test_large_outputs_have_their_own(ip):  # noqa: F811
    for name, call in outputs(ip, 4000, 1000).items():
        if name != "token_logprobs":
            out = call()
            assert len({t.untyped_storage().data_ptr() for t in out}) == len(out), name


def test_the_documents_say_so(ip):  # noqa: F811
    for f in (ip.quantize_fp4, ip.rmsnorm_i8, ip.token_logprobs):
        assert "share one storage" in " ".join(f.__doc__.split()), f.__name__
    assert "rmsnorm_i8" in ip.rmsnorm_fp4.__doc__
