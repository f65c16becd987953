"""Loading the library imports no torch: a process that only wants its constants or its C entry
points does not wait for one, and the native short forms are bound by the first call that may
take them (no GPU needed)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CONSTANTS = """
import sys, paper_2609_30846_gb300 as ip
ip.load()
assert ip.workspace_bytes(1, 8, 64) == 256 and ip.kv4_page_bytes(16) == 2304 and ip.dyadic_multiplier(0.5)
assert "torch" not in sys.modules
"""
FIRST_CALL = """
import sys, paper_2609_30846_gb300 as ip
ip.load()
pending = ip._short
import torch
for i in range(2):
    try:
        ip.quantize_rows_i8(torch.zeros(2, 16))
    except TypeError as exc:
        assert "CUDA tensor" in str(exc)
    else:
        raise AssertionError
    assert ip._short is not pending and ip._short is not ip._Unbound
assert pending.bind is ip._short.bind
"""


def run(code):
    env = dict(os.environ, PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-W", "error", "-c", code], env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]


def test_constants_need_no_torch():
    run(CONSTANTS)


def test_the_first_call_binds_the_short_forms():
    pytest.importorskip("torch")
    from paper_2609_30846_gb300 import _build
    if _build.torch_extension() is None:
        pytest.skip("no torch with CUDA to build for")
    run(FIRST_CALL)
