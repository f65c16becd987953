"""Row strides that the native short form of the scaled product reads from a tensor, on CPU tensors:
those of the general form, and none where the general form refuses the tensor."""
import importlib.util
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2609_30846_gb300 import _as_rows, _build

HARNESS = """
#include "%s"
namespace {
PyObject *py_row_stride(PyObject *, PyObject *t) {
    HANDLE_TH_ERRORS
    return PyLong_FromLongLong(row_stride(THPVariable_Unpack(t)));
    END_HANDLE_TH_ERRORS
}
PyMethodDef h_methods[] = {{"row_stride", py_row_stride, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef h_module = {PyModuleDef_HEAD_INIT, "harness", nullptr, -1, h_methods, nullptr, nullptr, nullptr, nullptr};
}
extern "C" PyObject *PyInit_harness() { return PyModule_Create(&h_module); }
"""


@pytest.fixture(scope="module")
def row_stride(tmp_path_factory):
    if _build._torch_dir() is None:
        pytest.skip("no torch with CUDA to build for")
    d = tmp_path_factory.mktemp("strides")
    src, out = str(d / "harness.cpp"), str(d / "harness.so")
    with open(src, "w") as f:
        f.write(HARNESS % _build.TORCH_SOURCE)
    cmd = [src if a == _build.TORCH_SOURCE else a for a in _build.torch_command(out)]
    subprocess.run(cmd, check=True, cwd=os.path.dirname(src))
    spec = importlib.util.spec_from_file_location("harness", out)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod.row_stride


def i8(*shape):
    return torch.zeros(*shape, dtype=torch.int8)


CASES = {
    "matrix": lambda: i8(4, 64), "row": lambda: i8(1, 64), "vector": lambda: i8(64), "odd row": lambda: i8(1, 33),
    "sliced rows": lambda: i8(4, 80)[:, :64], "sliced row": lambda: i8(4, 80)[1:2, 3:67],
    "transposed": lambda: i8(64, 4).t(), "row of a transposed": lambda: i8(64, 8).t()[:1],
    "step vector": lambda: i8(128)[::2], "step row": lambda: i8(1, 128)[:, ::2], "step row of many": lambda: i8(3, 128)[1:2, ::2],
    "one byte": lambda: i8(1, 1).expand(1, 64), "one byte vector": lambda: i8(1).expand(64),
    "expanded rows": lambda: i8(1, 64).expand(4, 64), "one column": lambda: i8(64, 1)[:1], "step column": lambda: i8(5, 32)[:, ::32],
    "element": lambda: i8(1, 128)[:, ::128], "three": lambda: i8(2, 3, 64), "three, one row": lambda: i8(4, 5, 64)[:1, 2:3],
    "three, one step row": lambda: i8(4, 5, 64)[:1, 2:3, ::2], "three, swapped": lambda: i8(2, 3, 64).transpose(0, 1),
    "no rows": lambda: i8(0, 64), "no rows, step": lambda: i8(0, 128)[:, ::2],
}


@pytest.mark.parametrize("name", list(CASES))
def test_the_general_forms_stride_or_none(row_stride, name):
    t = CASES[name]()
    try:
        want = _as_rows(t, "t")[2]
    except ValueError:
        want = None
    got = row_stride(t)
    if want is None:
        assert got < t.shape[-1]      # taken by the general form, which refuses it
    else:
        assert got in (want, 0) or t.numel() == 0
