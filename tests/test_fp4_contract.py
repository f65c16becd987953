"""What the product of 4-bit rows may be given, where a user reads it: the tensor cores' block scales have no
sign, so a negative one, which the values of rows take, would give an answer that goes by the sizes."""
import os
import re

import pytest

import paper_2609_30846_gb300 as ip

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def words(text):
    return " ".join(re.sub(r"^ \* ?", "", line) for line in text.splitlines()).replace("  ", " ")


def test_the_product_s_scales_are_from_zero_on():
    header = words(open(os.path.join(ROOT, "include", "ip_mhsa.h")).read())
    assert "any s but NaN" not in header
    assert "any s from 0 on but NaN (bytes 0 to 0x7e)" in header and "so ip_linear_fp4's must not" in header
    assert "Block scales are from 0 on (bytes 0 to 0x7e" in words(ip.linear_fp4.__doc__)


def test_what_the_library_writes_is_allowed():
    # of the definition's own bytes (tests/fp4_ref.py), which the calls give bit for bit, none has a sign or is NaN
    torch = pytest.importorskip("torch")
    import fp4_ref as ref
    g = torch.Generator().manual_seed(1)
    x = torch.randn(64, 200, generator=g) * torch.exp(4 * torch.randn(64, 200, generator=g))
    sb = ref.quantize(x)[1]
    assert int(sb.max()) <= 0x7e and sb.dtype == torch.uint8
